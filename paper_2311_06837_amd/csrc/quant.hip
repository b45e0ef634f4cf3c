// Rows and weights on the 8-bit grid of gnn_linear_i8_fwd.
//   a = max_k |x_k|,   scale = a / 127,   q_k = the whole number nearest to 127 x_k / a (ties to even)
// The largest code is 127 on either side, so a sum of products of codes is symmetric and -128 never appears.
// Which code is the nearest is decided exactly: a float that lands within 2e-5 of a border between two codes in 32 bits (one in 25 000; eight
// at a time) is divided again in 64 bits, where 127 x is exact and the quotient of two floats cannot round across a border.  bfloat16
// never needs that (see codes_of).
// A row below 2^-120 becomes zeros (127 / a would not be finite); a row that holds an infinity or NaN gets the scale NaN and
// codes 0, so that it stays NaN in whatever is computed from it and no other row is touched.
#include "quant.h"

namespace gnnhot {

// ---- rows ----------------------------------------------------------------------------------------------------------
// LR lanes own a row; lane sl holds the groups of eight sl, sl + LR, ... of it in registers (NV of them): one read of the row, one store
// of its codes.  LR and NV are picked so that few lanes idle beyond the row's end (602 columns are 76 groups: 16 lanes x 5).  Bound: HBM.  With the values written too: 1M rows of 1024 bfloat16 890 to 900 us (860 to 1000 by the card; 5.1 to 6 TB/s),
// 186 000 listed rows of 602 floats, whose rows start on 8 bytes only, 278 us (235 to 280; 3.6 to 4.3 TB/s).
template <int DT, int LR, int NV, int AL>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantRows a) {
    constexpr int RPW = 64 / LR;
    const int lane = lane_id(), sl = lane % LR;
    const int64_t wave = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 6, n_waves = (int64_t)gridDim.x * 4;
    const int K = a.K, Kq = (K + 15) & ~15;
    for (int64_t base = wave * RPW; base < a.n_active; base += n_waves * RPW) {   // uniform over the wavefront
        const int64_t i = base + lane / LR;
        const bool active = i < a.n_active;
        const int64_t v = active ? (a.rows ? (int64_t)a.rows[i] : i) : 0;
        const int64_t o = a.compact ? i : v;
        Raw8<DT> raw[NV];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k) raw[k] = load_raw8<DT, AL>(a.X, v * a.ldx, (sl + LR * k) * 8, active ? K : 0);
#pragma unroll
        for (int k = 0; k < NV; ++k) top = raw[k].largest(top);
        const RowGrid g = row_grid(group_max<LR>(Raw8<DT>::whole_pattern(top)));
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int c0 = (sl + LR * k) * 8;
            if (active && c0 < Kq) {
                float x[8];
                raw[k].to_float(x);
                *(uint2*)(a.Q + o * a.ldq + c0) = codes_of<DT>(x, g);
                if (a.values) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = x[e] * g.scale;
                    store8<DT, AL>(a.values, v * a.ldv, c0, K, x);
                }
            }
        }
        if (active && sl == 0) a.scale[o] = g.scale;
    }
}

// Rows too long for one wavefront's registers: a workgroup a row, read twice (the second time from the caches).
template <int DT, int AL>
__global__ __launch_bounds__(256) void quantize_long_rows_kernel(QuantRows a) {
    __shared__ uint32_t s_top[4];
    const int K = a.K, Kq = (K + 15) & ~15;
    for (int64_t i = blockIdx.x; i < a.n_active; i += gridDim.x) {   // uniform over the workgroup
        const int64_t v = a.rows ? (int64_t)a.rows[i] : i, o = a.compact ? i : v;
        uint32_t top = 0;
        for (int c0 = threadIdx.x * 8; c0 < K; c0 += 2048) {
            float x[8];
            load8<DT, AL>(a.X, v * a.ldx, c0, K, x);
            top = largest_pattern(x, top);
        }
        top = wave_max_u32(top);
        __syncthreads();
        if (lane_id() == 0) s_top[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) top = s_top[w] > top ? s_top[w] : top;
        const RowGrid g = row_grid(top);
        for (int c0 = threadIdx.x * 8; c0 < Kq; c0 += 2048) {
            float x[8];
            load8<DT, AL>(a.X, v * a.ldx, c0, K, x);
            *(uint2*)(a.Q + o * a.ldq + c0) = codes_of<DT>(x, g);
            if (a.values) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * g.scale;
                store8<DT, AL>(a.values, v * a.ldv, c0, K, x);
            }
        }
        if (threadIdx.x == 0) a.scale[o] = g.scale;
    }
}

template <int DT, int AL>
static int32_t launch_rows(const QuantRows& a, hipStream_t stream) {
    const int need = (a.K + 15) / 16 * 2;    // groups of a row; the codes up to a multiple of 16 are written too
#define GNN_QR(LR_, NV_)                                                                                                    \
    do {                                                                                                                    \
        quantize_rows_kernel<DT, LR_, NV_, AL><<<grid_for(a.n_active, 4 * (64 / LR_)), 256, 0, stream>>>(a);          \
        GNN_LAUNCH_CHECK("quantize_rows_kernel");                                                                           \
        return GNN_OK;                                                                                                      \
    } while (0)
    if (need <= 8) GNN_QR(8, 1);
    if (need <= 16) GNN_QR(16, 1);
    if (need <= 32) GNN_QR(16, 2);
    if (need <= 48) GNN_QR(16, 3);
    if (need <= 64) GNN_QR(32, 2);
    if (need <= 80) GNN_QR(16, 5);
    if (need <= 96) GNN_QR(32, 3);
    if (need <= 128) GNN_QR(64, 2);
    if (need <= 192) GNN_QR(64, 3);
    if (need <= 256) GNN_QR(64, 4);
    if (need <= 384) GNN_QR(64, 6);
    if (need <= 512) GNN_QR(64, 8);
#undef GNN_QR
    quantize_long_rows_kernel<DT, AL><<<grid_for(a.n_active, 1, 8192), 256, 0, stream>>>(a);
    GNN_LAUNCH_CHECK("quantize_long_rows_kernel");
    return GNN_OK;
}

template <int DT>
static int32_t launch_rows_aligned(const QuantRows& a, hipStream_t stream) {
    constexpr int es = DT == GNN_F32 ? 4 : 2;
    int al = row_alignment<DT>(a.X, a.ldx);
    if (a.values) al = al < row_alignment<DT>(a.values, a.ldv) ? al : row_alignment<DT>(a.values, a.ldv);
    if (al == 16) return launch_rows<DT, 16>(a, stream);
    return al == es ? launch_rows<DT, es>(a, stream) : launch_rows<DT, 2 * es>(a, stream);
}

int32_t quantize_rows(const QuantRows& a, int32_t dtype, hipStream_t stream) {
    return dtype == GNN_F32 ? launch_rows_aligned<GNN_F32>(a, stream) : launch_rows_aligned<GNN_BF16>(a, stream);
}

// ---- weights -------------------------------------------------------------------------------------------------------
// Two launches, so that the reduction over K is spread over the chip: largest bit pattern of each column over kSplitK rows, then
// the grid of each column from its few partial maxima, codes and layout (the second read comes from the caches).  4096 x 1031 floats with values
// 8.3 + 13.3 us: bound by latency, a chain of two dependent loads a launch.
constexpr int kSplitK = 64;

template <int DT>
__global__ __launch_bounds__(256) void column_top_kernel(const void* __restrict__ W, int64_t ldw, int32_t K, int32_t N, uint32_t* __restrict__ part) {
    __shared__ uint32_t s[4][64];
    const int n = (int)blockIdx.x * 64 + lane_id(), w = (int)threadIdx.x >> 6;
    const int k0 = (int)blockIdx.y * kSplitK, k1 = k0 + kSplitK < K ? k0 + kSplitK : K;
    uint32_t top = 0;
    if (n < N) {
        float x[kSplitK / 4];
#pragma unroll
        for (int j = 0; j < kSplitK / 4; ++j) x[j] = k0 + w + 4 * j < k1 ? load_one<DT>(W, (int64_t)(k0 + w + 4 * j) * ldw + n) : 0.f;
        top = largest_pattern(x, 0u);
    }
    s[w][lane_id()] = top;
    __syncthreads();
    if (w == 0 && n < N) {
#pragma unroll
        for (int j = 1; j < 4; ++j) top = s[j][lane_id()] > top ? s[j][lane_id()] : top;
        part[(int64_t)blockIdx.y * N + n] = top;
    }
}

// A thread makes the 16 bytes of one column and 16 consecutive k; a workgroup 32 columns and 128 k, i.e. 4 KB of the layout in one piece.
template <int DT>
__global__ __launch_bounds__(256) void pack_weight_kernel(const void* __restrict__ W, int64_t ldw, int32_t K, int32_t N, const uint32_t* __restrict__ part,
                                                          int32_t splits, int8_t* __restrict__ Wq, float* __restrict__ scale,
                                                          void* __restrict__ values, int64_t ldv) {
    __shared__ uint32_t s[8][32];
    const int col = (int)threadIdx.x % 32, grp = (int)threadIdx.x / 32, n = (int)blockIdx.x * 32 + col;
    const int k16 = (int)blockIdx.y * 8 + grp, n16 = (K + 63) / 64 * 4;
    float q[2][8];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int k = k16 * 16 + e;
        q[e / 8][e % 8] = k < K && n < N ? load_one<DT>(W, (int64_t)k * ldw + n) : 0.f;
    }
    uint32_t top = 0;
    if (n < N)
        for (int j = grp; j < splits; j += 8) {
            const uint32_t b = part[(int64_t)j * N + n];
            top = b > top ? b : top;
        }
    s[grp][col] = top;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) top = s[j][col] > top ? s[j][col] : top;
    if (k16 >= n16) return;
    const RowGrid g = row_grid(top);
    const uint2 lo = codes_of<DT>(q[0], g), hi = codes_of<DT>(q[1], g);
    *(uint4*)(Wq + (((int64_t)blockIdx.x * n16 + k16) * 32 + col) * 16) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    if (n >= N) return;
    if (values) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int k = k16 * 16 + e;
            if (k < K) store_one<DT>(values, (int64_t)k * ldv + n, q[e / 8][e % 8] * g.scale);
        }
    }
    if (k16 == 0) scale[n] = g.scale;
}

}  // namespace gnnhot

using namespace gnnhot;

extern "C" int32_t gnn_quantize_rows(const int32_t* rows, int32_t n_active, const void* X, int64_t ldx, int32_t K, int32_t dtype, int8_t* Q, int64_t ldq,
                                     float* scale, void* values, int64_t ldv, void* stream) {
    GNN_REQUIRE(n_active >= 0, GNN_ERR_INVALID_ARG, "negative row count");
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    GNN_REQUIRE(K >= 1, GNN_ERR_INVALID_ARG, "K = %d", K);
    GNN_REQUIRE(K <= kMaxI8K, GNN_ERR_UNSUPPORTED, "K = %d is over %d", K, kMaxI8K);
    GNN_REQUIRE(ldx >= K && (values == nullptr || ldv >= K), GNN_ERR_SHAPE, "leading dimension smaller than K");
    GNN_REQUIRE(ldq >= (K + 15) / 16 * 16 && ldq % 16 == 0, GNN_ERR_SHAPE, "ldq = %lld: a multiple of 16 of at least K = %d is needed", (long long)ldq, K);
    if (n_active == 0) return GNN_OK;
    GNN_REQUIRE(X != nullptr && Q != nullptr && scale != nullptr, GNN_ERR_INVALID_ARG, "X, Q or scale is NULL");
    GNN_REQUIRE(((uintptr_t)Q & 15u) == 0, GNN_ERR_INVALID_ARG, "Q is not 16-byte aligned");
    const QuantRows a = {rows, n_active, X, ldx, K, Q, ldq, scale, values, ldv, false};
    return quantize_rows(a, dtype, (hipStream_t)stream);
}

extern "C" int32_t gnn_quantize_weight(const void* W, int64_t ldw, int32_t K, int32_t N, int32_t dtype, int8_t* Wq, float* scale, void* values,
                                       int64_t ldv, void* ws, size_t* ws_bytes, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    GNN_REQUIRE(K >= 1 && N >= 1, GNN_ERR_INVALID_ARG, "K = %d, N = %d", K, N);
    GNN_REQUIRE(K <= kMaxI8K && N <= kMaxI8N, GNN_ERR_UNSUPPORTED, "K = %d, N = %d are over %d, %d", K, N, kMaxI8K, kMaxI8N);
    GNN_REQUIRE(ldw >= N && (values == nullptr || ldv >= N), GNN_ERR_SHAPE, "leading dimension smaller than N");
    const int splits = (K + kSplitK - 1) / kSplitK;
    WsCarver carve(ws);
    uint32_t* part = carve.take<uint32_t>((size_t)splits * N);
    bool query;
    GNN_CHECK(ws_protocol(ws, ws_bytes, carve.used, &query));
    if (query) return GNN_OK;
    GNN_REQUIRE(W != nullptr && Wq != nullptr && scale != nullptr, GNN_ERR_INVALID_ARG, "W, Wq or scale is NULL");
    GNN_REQUIRE(((uintptr_t)Wq & 15u) == 0, GNN_ERR_INVALID_ARG, "Wq is not 16-byte aligned");
    const dim3 g1((N + 63) / 64, splits), g2((N + 31) / 32, (K + 127) / 128);
    if (dtype == GNN_F32) {
        column_top_kernel<GNN_F32><<<g1, 256, 0, stream>>>(W, ldw, K, N, part);
        pack_weight_kernel<GNN_F32><<<g2, 256, 0, stream>>>(W, ldw, K, N, part, splits, Wq, scale, values, ldv);
    } else {
        column_top_kernel<GNN_BF16><<<g1, 256, 0, stream>>>(W, ldw, K, N, part);
        pack_weight_kernel<GNN_BF16><<<g2, 256, 0, stream>>>(W, ldw, K, N, part, splits, Wq, scale, values, ldv);
    }
    GNN_LAUNCH_CHECK("pack_weight_kernel");
    return GNN_OK;
}
