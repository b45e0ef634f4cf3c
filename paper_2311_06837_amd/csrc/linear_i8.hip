// Feature transform of a layer in 8-bit integers: the answers of a trained model.
//   H[v, n] = act( sA[v] wN[n] sum_k qA[v, k] qN[k, n]  (+ sX[v] wS[n] sum_k qX[v, k] qS[k, n]) + bias[n] )
// The sums over k are exact in int32; scales, bias and activation are applied in float.
//
// v_mfma_i32_32x32x32_i8 with the operands exchanged: the weights are the first operand, so a lane holds four CONSECUTIVE columns of one
// row of the output and its row scale is one register.
#include "quant.h"

namespace gnnhot {

// Products and sums of the scales are rounded one by one in every kernel of this file: a row's answer is the same to the bit whichever of
// them runs, however its inputs come and however many rows are asked for with it.
#pragma clang fp contract(off)

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void glb_void;

struct LinearI8 {
    const int32_t* rows;         // of the output
    const int32_t* in_rows;      // of the inputs: rows, or NULL where their codes were made by this call in list order
    int32_t n_active;
    const void* A[2];
    const float* sa[2];
    int64_t lda;
    int32_t K;
    const int8_t* W[2];
    const float* sw[2];
    const float* bias;
    int32_t N;
    void* H;
    int64_t ldh;
    int32_t relu;
    int32_t n_src;
    int64_t tiles_m;
    int32_t tiles_n;
    bool vec_out, vec_out8;   // four, eight columns of the output are aligned to their bytes
    int32_t out_dtype;
};

// ids are dealt round-robin over the 8 XCDs: consecutive tiles of one XCD share its L2.  Grid: 8 * ceil(total / 8).
__device__ __forceinline__ int64_t xcd_tile(int64_t id, int64_t total) {
    const int64_t per = (total + 7) / 8;
    return (id % 8) * per + id / 8;
}

__device__ __forceinline__ void copy_to_lds(const void* g, void* l) {
    __builtin_amdgcn_global_load_lds((glb_void*)g, (lds_void*)l, 16, 0, 0);
}

// Four columns n .. n + 3 of output row v.
template <int OUT>
__device__ __forceinline__ void store_four(const LinearI8& a, int64_t v, int n, float (&y)[4]) {
    if (a.relu) {
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = y[e] < 0.f ? 0.f : y[e];     // NaN stays
    }
    const int64_t o = v * a.ldh + n;
    if (a.vec_out && n + 3 < a.N) {
        if (OUT == GNN_F32) *(float4*)((float*)a.H + o) = make_float4(y[0], y[1], y[2], y[3]);
        else *(uint2*)((uint16_t*)a.H + o) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) store_one<OUT>(a.H, o + e, y[e]);
    }
}

// A lane's 16 columns of a block of 32 x 32: 8 q + 4 (lane / 32) + 0 .. 3 of output row v, which is one of the call's.
template <int OUT>
__device__ __forceinline__ void store_block(const LinearI8& a, int64_t v, int n0, float (&y)[16]) {
    if (OUT == GNN_BF16 && a.vec_out8 && n0 + 32 <= a.N) {
        if (a.relu) {
#pragma unroll
            for (int k = 0; k < 16; ++k) y[k] = y[k] < 0.f ? 0.f : y[k];     // NaN stays
        }
        // the halves of the wavefront trade words: eight columns in a row, 16 bytes, for every lane (both halves hold the same rows,
        // so both of a pair are here or neither is)
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            uint32_t w0[2], w1[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const auto s = __builtin_amdgcn_permlane32_swap(pack_bf16(y[4 * q + 2 * e], y[4 * q + 2 * e + 1]),
                                                                pack_bf16(y[4 * q + 4 + 2 * e], y[4 * q + 4 + 2 * e + 1]), false, false);
                w0[e] = s[0];
                w1[e] = s[1];
            }
            *(uint4*)((uint16_t*)a.H + v * a.ldh + n0 + 8 * q + 8 * (lane_id() / 32)) = make_uint4(w0[0], w0[1], w1[0], w1[1]);
        }
        return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int n = n0 + 8 * q + 4 * (lane_id() / 32);
        if (n >= a.N) continue;
        float four[4] = {y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
        store_four<OUT>(a, v, n, four);
    }
}

// A barrier that leaves the wavefront's LATER youngest loads on their way (they return in order; all its LDS reads are done).  The one of
// __syncthreads, and of a fence for LDS alone, waits for every load that fills LDS.
template <int LATER>
__device__ __forceinline__ void slice_barrier() {
    __builtin_amdgcn_s_waitcnt(0x0070 | (LATER & 15) | (LATER >> 4) << 14);
    asm volatile("s_barrier" ::: "memory");
}

// ---- tile kernel ------------------------------------------------------------------------------------------------------
// Long reductions: WM x WN wavefronts, each MT x NT blocks of 32 x 32 of the output.  The reduction moves in slices of 64 bytes through a ring
// of R LDS buffers that the loads fill themselves (no registers in between): R - 1 slices are on their way or being multiplied, one
// barrier a slice.  With two buffers of 128 bytes every slice waited for loads that had been asked for during the one before: 33 % of
// the wavefronts' time, 8192 x 4096 x 4096 in 175 to 185 us whatever the tile.  Now 129 to 140 us by the card, 2.0 to 2.1 POP/s (a large bfloat16 product of the
// library runs at 1.19 PFLOP/s).  Bound by the operands' way through LDS: for 32 of the
// reduction a workgroup reads 48 KB of it (384 clocks) and multiplies for 512, and the loads that fill it want the same port.
// A row's 64 bytes are stored with their 16-byte chunk c at slot c ^ ((row >> 2) & 3), by choosing which chunk a lane asks for: sixteen
// consecutive rows read with the same c touch all 64 banks once.  The weights come in the order of the instruction's lanes.
template <int OUT, int MT, int NT, int WM, int WN, int R, bool TWO>
__global__ __launch_bounds__(64 * WM * WN) void linear_i8_kernel(LinearI8 a) {
    constexpr int NW = WM * WN, BM = 32 * MT * WM, BNB = NT * WN;   // rows, blocks of 32 columns
    constexpr int A_BYTES = BM * 64, B_BYTES = BNB * 2048, STAGE = A_BYTES + B_BYTES;
    constexpr int PA = BM / 16 / NW, PB = BNB * 2 / NW;             // pieces of 1 KB a wavefront moves in a slice
    constexpr int SRC = TWO ? 2 : 1;
    static_assert(PA * NW * 16 == BM && PB * NW == BNB * 2, "pieces divide");
    extern __shared__ __attribute__((aligned(64))) int8_t codes[];
    __shared__ __attribute__((aligned(16))) float s_w[SRC][BNB * 32], s_b[BNB * 32];
    const int64_t total = a.tiles_m * a.tiles_n;
    const int64_t tile = xcd_tile(blockIdx.x, total);
    if (tile >= total) return;
    // four rows of tiles, column by column: the tiles that an XCD has at a time share more of their rows and weights in its L2
    const int64_t group = tile / (4 * (int64_t)a.tiles_n), within = tile - group * 4 * a.tiles_n;
    const int high = a.tiles_m - 4 * group < 4 ? (int)(a.tiles_m - 4 * group) : 4;
    const int64_t tm = 4 * group + within % high;
    const int tn = __builtin_amdgcn_readfirstlane((int)(within / high));
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int64_t m0 = tm * BM;
    const int nb0 = tn * BNB, nb_all = (a.N + 31) / 32;
    const int n16 = (a.K + 63) / 64 * 4, slices = n16 / 4, Kr = (a.K + 15) & ~15;

    int64_t row_off[PA];
    int chunk[PA];
#pragma unroll
    for (int p = 0; p < PA; ++p) {
        const int r = (p * NW + wave) * 16 + lane / 4;
        int64_t i = m0 + r;
        if (i >= a.n_active) i = a.n_active - 1;      // computed and dropped
        row_off[p] = (a.in_rows ? (int64_t)a.in_rows[i] : i) * a.lda;
        chunk[p] = ((lane & 3) ^ ((r >> 2) & 3)) * 16;
    }
    int64_t b_off[PB];
#pragma unroll
    for (int p = 0; p < PB; ++p) {
        const int q = p * NW + wave;
        int nb = nb0 + q / 2;
        if (nb >= nb_all) nb = nb_all - 1;
        b_off[p] = (int64_t)nb * n16 * 512 + (q % 2) * 1024 + lane * 16;
    }
    // The nth slice of the call (those of the second source follow on); beyond the end the last one again, which nobody reads: every
    // wavefront has the same number of loads on its way in every slice, and waits by counting them.
    const auto fetch = [&](int nth, int8_t* to) {
        const int n = nth < SRC * slices ? nth : SRC * slices - 1, s = TWO && n >= slices ? n - slices : n;
        const int8_t* A = (const int8_t*)(TWO && n >= slices ? a.A[1] : a.A[0]);
        const int8_t* W = TWO && n >= slices ? a.W[1] : a.W[0];
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int k = s * 64 + chunk[p];
            copy_to_lds(A + row_off[p] + (k < Kr ? k : s * 64), to + (p * NW + wave) * 1024);    // beyond K the weights are zeros
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) copy_to_lds(W + b_off[p] + (int64_t)s * 2048, to + A_BYTES + (p * NW + wave) * 1024);
    };
    for (int c = threadIdx.x; c < BNB * 32; c += 64 * NW) {
        const int n = nb0 * 32 + c < a.N ? nb0 * 32 + c : 0;
        s_w[0][c] = a.sw[0][n];
        if (TWO) s_w[SRC - 1][c] = a.sw[1][n];
        s_b[c] = a.bias ? a.bias[n] : 0.f;
    }
    int64_t out_row[MT];
    float s_row[SRC][MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t r = m0 + (wm * MT + i) * 32 + (lane & 31), c = r < a.n_active ? r : a.n_active - 1;
        out_row[i] = r < a.n_active ? (a.rows ? (int64_t)a.rows[c] : c) : -1;
        const int64_t v = a.in_rows ? (int64_t)a.in_rows[c] : c;
        s_row[0][i] = a.sa[0][v];
        if (TWO) s_row[SRC - 1][i] = a.sa[1][v];
    }

    v16i acc[MT][NT];
    float sum[TWO ? MT : 1][TWO ? NT : 1][16];
    const v16i zero = {};
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = zero;
    const int a_at = (wm * MT * 32 + (lane & 31)) * 64, b_at = A_BYTES + wn * NT * 2048 + lane * 16;
    const int swz = (lane >> 2) & 3;     // (row >> 2) & 3: blocks of 32 rows leave it alone

#pragma unroll
    for (int r = 0; r < R - 1; ++r) fetch(r, codes + r * STAGE);
    int at = 0, free_at = (R - 1) * STAGE;
#pragma unroll
    for (int src = 0; src < SRC; ++src) {
        for (int s = 0; s < slices; ++s) {
            // all but the loads of the R - 2 youngest slices have arrived (they return in order), for every wavefront
            slice_barrier<(R - 2) * (PA + PB)>();
            const int8_t* l = codes + at;
            v4i fa[2][MT], fb[2][NT];
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
                for (int j = 0; j < NT; ++j) fb[kk][j] = *(const v4i*)(l + b_at + j * 2048 + kk * 1024);
#pragma unroll
                for (int i = 0; i < MT; ++i) fa[kk][i] = *(const v4i*)(l + a_at + i * 2048 + ((2 * kk + lane / 32) ^ swz) * 16);
            }
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                // the next slice is asked for between the two steps: before the first its loads hold up the fragments' (135 us against 129)
                if (kk == 1) fetch(src * slices + s + R - 1, codes + free_at);     // where the slice before this one was: everybody has read it
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[kk][j], fa[kk][i], acc[i][j], 0, 0, 0);
            }
            free_at = at;
            at = at + STAGE < R * STAGE ? at + STAGE : 0;
        }
        if (TWO && src == 0) {
            // the neighbour half, scaled, waits in float for the vertex's own
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 w = *(const float4*)&s_w[0][(wn * NT + j) * 32 + 8 * q + 4 * (lane / 32)];
                    const float we[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            sum[TWO ? i : 0][TWO ? j : 0][4 * q + e] = (float)acc[i][j][4 * q + e] * (s_row[0][i] * we[e]);
                            acc[i][j][4 * q + e] = 0;
                        }
                }
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);   // the loads beyond the end have landed: they write to this workgroup's LDS

#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int n0 = (nb0 + wn * NT + j) * 32;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            float y[16];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = (wn * NT + j) * 32 + 8 * q + 4 * (lane / 32);
                const float4 w = *(const float4*)&s_w[SRC - 1][c], b = *(const float4*)&s_b[c];
                const float we[4] = {w.x, w.y, w.z, w.w}, be[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[4 * q + e] = (float)acc[i][j][4 * q + e] * (s_row[SRC - 1][i] * we[e]);
                    if (TWO) y[4 * q + e] = sum[TWO ? i : 0][TWO ? j : 0][4 * q + e] + y[4 * q + e];
                    y[4 * q + e] += be[e];
                }
            }
            if (out_row[i] >= 0) store_block<OUT>(a, out_row[i], n0, y);
        }
    }
}

template <int OUT, int MT, int NT, int WM, int WN, int R, bool TWO>
static int32_t launch_tile(LinearI8 a, hipStream_t stream) {
    constexpr int BM = 32 * MT * WM, BN = 32 * NT * WN, bytes = R * (BM + BN) * 64;
    a.tiles_m = ((int64_t)a.n_active + BM - 1) / BM;
    a.tiles_n = (a.N + BN - 1) / BN;
    const int64_t total = a.tiles_m * a.tiles_n;
    GNN_REQUIRE(total < ((int64_t)1 << 30), GNN_ERR_UNSUPPORTED, "too many output tiles");
    const void* kernel = (const void*)linear_i8_kernel<OUT, MT, NT, WM, WN, R, TWO>;
    if (bytes > 48 * 1024) GNN_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    linear_i8_kernel<OUT, MT, NT, WM, WN, R, TWO><<<(int)((total + 7) / 8 * 8), 64 * WM * WN, bytes, stream>>>(a);
    GNN_LAUNCH_CHECK("linear_i8_kernel");
    return GNN_OK;
}

// ---- panel kernel -----------------------------------------------------------------------------------------------------
// Many rows of at most 1024 columns, the shape of a graph's layers: tiles of 32 or 64 rows, and a panel of up to 512 output columns.
// The rows are read once, as they come (codes, or floats that are put on the grid on the way: the row's largest, then its codes, without
// a trip through memory), and lie in LDS in the order of the instruction's lanes, both sources side by side; the weights come
// straight from L2 into registers, four steps ahead.  Bound: HBM, by the rows as they come.
// A workgroup of 16 wavefronts has a CU to itself and stays for many tiles.  Eight of them fetch the rows of the next tile and put them on
// the grid, eight multiply this tile, and they meet at one barrier a tile.  With every wavefront doing both in turn and
// two workgroups on a CU all read at once and then all multiplied at once: 602 + 602 bfloat16 columns to 256, 186 000 rows, took the
// sum of the two (95 us to read, 53 to multiply, 41 to store).  Now 158 to 171 us, 3.2 to 3.4 TB/s: the fetching half takes 120 us by itself (two of its wavefronts
// a SIMD, 70 us of it arithmetic), the multiplying half 88.  No unit is full (vector 45 %, matrix 15 %): wavefronts wait for 62 % of their time, for
// rows and at the barrier, and which of the two was not told apart.
// LDS: two buffers of source, block of 32 rows, group of 16 k, row, 16 bytes; row r of group g at slot r ^ 4 (g mod 8), which spreads the groups of
// four rows that a wavefront writes at once, 512 bytes apart.  Conflicts are left: 1.96 clocks an LDS instruction, 6 % of a CU's clocks.
// Tiles of 64 rows keep 2 to 9 of 128 registers in scratch (12 to 40 bytes a lane); bfloat16 rows of 641 to 1024 columns that do not start on
// 16 bytes 30 to 136 (120 to 336 bytes).
constexpr int kPanelBlocks = 16;     // blocks of 32 columns a workgroup may have

template <int IN, int KC>
struct PanelRow {     // a lane's share of a row of one source, as it lies in memory
    Raw8<IN == GNN_F32 ? GNN_F32 : GNN_BF16> raw[KC];
};
template <int KC>
struct PanelRow<GNN_I8, KC> {
    uint4 q[(KC + 1) / 2];
    float scale;
};

// 16 lanes a row, eight columns a lane and step (codes: 16 of them)
template <int IN, int AL, int KC>
__device__ __forceinline__ void panel_fetch(const LinearI8& a, int s, int64_t v, int sl, PanelRow<IN, KC>& to) {
    if constexpr (IN == GNN_I8) {
        const int8_t* from = (const int8_t*)a.A[s] + v * a.lda;
#pragma unroll
        for (int k = 0; k < (KC + 1) / 2; ++k) {
            const int g = sl + 16 * k;      // beyond K: zeros (the weights are zeros there, too)
            to.q[k] = g * 16 < a.K ? *(const uint4*)(from + g * 16) : make_uint4(0u, 0u, 0u, 0u);
        }
        to.scale = a.sa[s][v];
    } else {
#pragma unroll
        for (int k = 0; k < KC; ++k) to.raw[k] = load_raw8<IN == GNN_F32 ? GNN_F32 : GNN_BF16, AL>(a.A[s], v * a.lda, (sl + 16 * k) * 8, a.K);
    }
}

// to LDS; the row's scale
template <int IN, int KC>
__device__ __forceinline__ float panel_stage(const PanelRow<IN, KC>& from, int8_t* to, int steps, int sl, int rr) {
    if constexpr (IN == GNN_I8) {
#pragma unroll
        for (int k = 0; k < (KC + 1) / 2; ++k) {
            const int g = sl + 16 * k;
            if (g < 2 * steps) *(uint4*)(to + g * 512 + ((rr ^ (4 * (g & 7))) & 31) * 16) = from.q[k];
        }
        return from.scale;
    } else {
        constexpr int DT = IN == GNN_F32 ? GNN_F32 : GNN_BF16;
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < KC; ++k) top = from.raw[k].largest(top);
        const RowGrid g = row_grid(group_max<16>(Raw8<DT>::whole_pattern(top)));
        int8_t* at = to + (sl / 2) * 512 + ((rr ^ (4 * ((sl / 2) & 7))) & 31) * 16 + (sl % 2) * 8;     // 16 lanes are 8 groups: the slot is the same in every step
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            float x[8];
            from.raw[k].to_float(x);
            if (sl + 16 * k < 4 * steps) *(uint2*)(at + k * 4096) = codes_of<DT>(x, g);
        }
        return g.scale;
    }
}

template <int IN, int AL, int KC, bool TWO, int MB>
__global__ __launch_bounds__(1024) void linear_i8_panel_kernel(LinearI8 a, int32_t panel_blocks) {
    extern __shared__ __attribute__((aligned(64))) int8_t codes[];
    constexpr int SRC = TWO ? 2 : 1;
    __shared__ __attribute__((aligned(16))) float s_row[2][2][32 * MB], s_w[2][kPanelBlocks * 32], s_b[kPanelBlocks * 32];
    // the panels of the same rows run next to each other on one XCD, and a workgroup keeps its panel
    // (quotients are computed in vector registers: back to scalar ones, where addresses made of them cost nothing)
    const int xcd = (int)blockIdx.x % 8, j = (int)blockIdx.x / 8, set = __builtin_amdgcn_readfirstlane(j / a.tiles_n);
    const int nb0 = (j - set * a.tiles_n) * panel_blocks;
    const int stride = __builtin_amdgcn_readfirstlane((int)gridDim.x / a.tiles_n), tile0 = set * 8 + xcd, tiles = (int)a.tiles_m;
    if (tile0 >= tiles) return;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int steps = (a.K + 31) / 32, block_bytes = steps * 1024, src_bytes = MB * block_bytes, buf_bytes = SRC * src_bytes;
    for (int c = threadIdx.x; c < panel_blocks * 32; c += 1024) {
        const int n = nb0 * 32 + c < a.N ? nb0 * 32 + c : 0;
        s_w[0][c] = a.sw[0][n];
        if (TWO) s_w[1][c] = a.sw[1][n];
        s_b[c] = a.bias ? a.bias[n] : 0.f;
    }

    if (wave < 8) {
        // units of 32 rows of one source; the next one or two are on their way, as many as a lane's registers hold
        constexpr int UNITS = MB * SRC, HELD = UNITS >= 2 && 2 * KC * (IN == GNN_F32 ? 8 : 4) <= 80 ? 2 : 1;
        const int sl = lane % 16, rr = wave * 4 + lane / 16;
        PanelRow<IN, KC> row[HELD];
        const auto fetch = [&](int tile, int u, PanelRow<IN, KC>& to) {
            const int64_t r = (int64_t)tile * (32 * MB) + (u % MB) * 32 + rr, i = r < a.n_active ? r : a.n_active - 1;     // computed and dropped
            panel_fetch<IN, AL, KC>(a, u / MB, a.in_rows ? (int64_t)a.in_rows[i] : i, sl, to);
        };
#pragma unroll
        for (int u = 0; u < HELD; ++u) fetch(tile0, u, row[u]);
        int buf = 0;
        for (int tile = tile0; tile < tiles; tile += stride, buf ^= 1) {     // uniform over the workgroup
            const int then = tile + stride < tiles ? tile + stride : tile;   // the last tile is fetched twice in part
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const float s = panel_stage<IN, KC>(row[u % HELD], codes + buf * buf_bytes + u * block_bytes, steps, sl, rr);
                if (sl == 0) s_row[buf][u / MB][(u % MB) * 32 + rr] = s;
                fetch(u + HELD < UNITS ? tile : then, (u + HELD) % UNITS, row[u % HELD]);
            }
            __syncthreads();     // this tile is whole, and the one before it has been multiplied
        }
        return;
    }

    constexpr int D = 4;     // steps of weights on their way; with it the slot of a row repeats: group 2 k + lane / 32 mod 8
    int at[D];
#pragma unroll
    for (int d = 0; d < D; ++d) {
        const int g = 2 * d + lane / 32;
        at[d] = g * 512 + ((lane ^ (4 * g)) & 31) * 16;
    }
    const int n16w = (a.K + 63) / 64 * 4;
    // The weights of a wavefront's blocks are one stream that starts over with every tile (block, source, step): what the next block,
    // source or tile begins with is fetched while this one ends.
    const auto weights = [&](int src, int b) -> const int8_t* { return (src == 0 ? a.W[0] : a.W[1]) + (int64_t)(nb0 + b) * n16w * 512; };
    const auto step_of = [&](const int8_t* w, int k) -> v4i { return *(const v4i*)(w + (k < steps ? k : steps - 1) * 1024 + lane * 16); };
    const int b_first = wave - 8;
    const bool busy = b_first < panel_blocks && (nb0 + b_first) * 32 < a.N;
    v4i fb[D];
    if (busy) {
#pragma unroll
        for (int d = 0; d < D; ++d) fb[d] = step_of(weights(0, b_first), d);
    }
    int buf = 0;
    for (int tile = tile0; tile < tiles; tile += stride, buf ^= 1) {     // uniform over the workgroup
        int64_t v[MB];
#pragma unroll
        for (int i = 0; i < MB; ++i) {
            const int64_t r = (int64_t)tile * (32 * MB) + 32 * i + lane % 32;
            v[i] = r < a.n_active ? (a.rows ? (int64_t)a.rows[r] : r) : -1;
        }
        __syncthreads();
        if (!busy) continue;
        for (int b = b_first;;) {
            const int b_next = b + 8 < panel_blocks && (nb0 + b + 8) * 32 < a.N ? b + 8 : b_first;
            const int n0 = (nb0 + b) * 32;
            float sum[MB][16] = {};
#pragma unroll 1
            for (int src = 0; src < SRC; ++src) {
                v16i acc[MB];
                const v16i zero = {};
#pragma unroll
                for (int i = 0; i < MB; ++i) acc[i] = zero;
                const int8_t* w = weights(src, b);
                const int8_t* wn = TWO && src == 0 ? weights(1, b) : weights(0, b_next);
                const int8_t* la = codes + buf * buf_bytes + src * src_bytes;
                int k0 = 0;
                for (; k0 + D <= steps; k0 += D) {      // without branches: the rows of one step are read while the step before is multiplied
                    const int8_t* wk = k0 + D < steps ? w + (k0 + D) * 1024 : wn;
                    const int most = k0 + D < steps ? steps - 1 - (k0 + D) : steps - 1;
                    v4i fa[2][MB];
#pragma unroll
                    for (int i = 0; i < MB; ++i) fa[0][i] = *(const v4i*)(la + i * block_bytes + k0 * 1024 + at[0]);
#pragma unroll
                    for (int d = 0; d < D; ++d) {
                        if (d + 1 < D)
#pragma unroll
                            for (int i = 0; i < MB; ++i) fa[(d + 1) & 1][i] = *(const v4i*)(la + i * block_bytes + k0 * 1024 + at[(d + 1) % D]);
#pragma unroll
                        for (int i = 0; i < MB; ++i) acc[i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[d], fa[d & 1][i], acc[i], 0, 0, 0);
                        fb[d] = *(const v4i*)(wk + (d < most ? d : most) * 1024 + lane * 16);
                    }
                }
                if (k0 < steps) {
#pragma unroll
                    for (int d = 0; d < D; ++d) {
                        if (k0 + d < steps)
#pragma unroll
                            for (int i = 0; i < MB; ++i)
                                acc[i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[d], *(const v4i*)(la + i * block_bytes + k0 * 1024 + at[d]), acc[i], 0, 0, 0);
                        fb[d] = step_of(wn, d);
                    }
                }
                const float* sw = s_w[src] + b * 32 + 4 * (lane / 32);
                float sr[MB];
#pragma unroll
                for (int i = 0; i < MB; ++i) sr[i] = s_row[buf][src][32 * i + lane % 32];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 f = *(const float4*)(sw + 8 * q);
#pragma unroll
                    for (int i = 0; i < MB; ++i) {      // the neighbour half first, then the vertex's own
                        sum[i][4 * q + 0] += (float)acc[i][4 * q + 0] * (sr[i] * f.x);
                        sum[i][4 * q + 1] += (float)acc[i][4 * q + 1] * (sr[i] * f.y);
                        sum[i][4 * q + 2] += (float)acc[i][4 * q + 2] * (sr[i] * f.z);
                        sum[i][4 * q + 3] += (float)acc[i][4 * q + 3] * (sr[i] * f.w);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < MB; ++i) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4 f = *(const float4*)(s_b + b * 32 + 8 * q + 4 * (lane / 32));
                    sum[i][4 * q + 0] += f.x;
                    sum[i][4 * q + 1] += f.y;
                    sum[i][4 * q + 2] += f.z;
                    sum[i][4 * q + 3] += f.w;
                }
                if (v[i] < 0) continue;
                if (a.out_dtype == GNN_F32) store_block<GNN_F32>(a, v[i], n0, sum[i]);
                else store_block<GNN_BF16>(a, v[i], n0, sum[i]);
            }
            b = b_next;
            if (b == b_first) break;
        }
    }
}

constexpr int kPanelLds = 155648;    // bytes of codes that leave room for the scales in 160 KB: 19 steps of 64 rows of two sources, twice

template <int IN, int AL, int KC, int MB>
static int32_t launch_panel_m(LinearI8 a, hipStream_t stream) {
    const int blocks = (a.N + 31) / 32;
    a.tiles_m = ((int64_t)a.n_active + 32 * MB - 1) / (32 * MB);
    // the widest panel that N fills, narrower ones as long as there are fewer tiles than compute units
    int panel = blocks < kPanelBlocks ? blocks : kPanelBlocks;
    while (panel > 2 && a.tiles_m * ((blocks + panel - 1) / panel) < 256) panel = (panel + 1) / 2;
    a.tiles_n = (blocks + panel - 1) / panel;
    const int bytes = 2 * MB * a.n_src * ((a.K + 31) / 32) * 1024;
    // a workgroup a CU, as many of each of the eight XCDs' tiles
    const int64_t rows8 = (a.tiles_m + 7) / 8, sets = 32 / a.tiles_n > 0 ? 32 / a.tiles_n : 1;
    const int grid = (int)(8 * (sets < rows8 ? sets : rows8) * a.tiles_n);
    const void* kernel = a.n_src == 2 ? (const void*)linear_i8_panel_kernel<IN, AL, KC, true, MB> : (const void*)linear_i8_panel_kernel<IN, AL, KC, false, MB>;
    if (bytes > 48 * 1024) GNN_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (a.n_src == 2) linear_i8_panel_kernel<IN, AL, KC, true, MB><<<grid, 1024, bytes, stream>>>(a, panel);
    else linear_i8_panel_kernel<IN, AL, KC, false, MB><<<grid, 1024, bytes, stream>>>(a, panel);
    GNN_LAUNCH_CHECK("linear_i8_panel_kernel");
    return GNN_OK;
}

template <int IN, int AL, int KC>
static int32_t launch_panel_k(const LinearI8& a, hipStream_t stream) {
    // tiles of 64 rows, whose weights are fetched half as often, where two of them fit and every CU has one
    const bool wide = 4 * a.n_src * ((a.K + 31) / 32) * 1024 <= kPanelLds && a.n_active >= 64 * 256;
    return wide ? launch_panel_m<IN, AL, KC, 2>(a, stream) : launch_panel_m<IN, AL, KC, 1>(a, stream);
}

template <int IN, int AL>
static int32_t launch_panel(const LinearI8& a, hipStream_t stream) {
    if (a.K <= 256) return launch_panel_k<IN, AL, 2>(a, stream);
    if constexpr (IN == GNN_I8) return launch_panel_k<IN, AL, 5>(a, stream);    // codes of more than 640 columns take tiles
    else return a.K <= 640 ? launch_panel_k<IN, AL, 5>(a, stream) : launch_panel_k<IN, AL, 8>(a, stream);
}

// ---- few rows -----------------------------------------------------------------------------------------------------------
// At most 32 rows: the weights are what is read, so a workgroup takes 16 columns only and its 8 wavefronts share the reduction, 64 k of every
// 512 each (v_mfma_i32_16x16x64_i8, weights straight into its lanes, four steps at once); the partial sums, whole numbers, meet in LDS in any
// order.  Rows that come as floats are put on the grid by every workgroup for itself where they are few: that is cheaper than a
// launch before this one.  One row of 602 + 602 floats to 256: 6.3 us, most of it the chain row, codes, weights, sum; 32 rows of
// codes 4096 -> 4096: 7.9 us, 2.1 TB/s of weights; 20 rows 602 + 602 -> 256: 10.7 us, 13.2 with the codes made in a launch before.
constexpr int kFewRows = 32;
constexpr int kFewCodes = 49152;    // bytes of LDS for codes made here

template <int IN, int AL, int MT, bool TWO>
__global__ __launch_bounds__(512) void linear_i8_few_kernel(LinearI8 a) {
    constexpr int SRC = TWO ? 2 : 1;
    constexpr int RED = 8 * MT * SRC * 1024;
    __shared__ __attribute__((aligned(16))) int8_t lds[IN == GNN_I8 || RED > kFewCodes ? RED : kFewCodes];
    __shared__ float s_row[SRC][kFewRows];
    const int lane = lane_id(), wave = (int)threadIdx.x >> 6;
    const int K = a.K, n16w = (K + 63) / 64 * 4, steps = n16w / 4, M = a.n_active;
    const int n0 = (int)blockIdx.x * 16;
    const int col = lane % 16, kg = lane / 16;
    v4i acc[SRC][MT];
#pragma unroll
    for (int s = 0; s < SRC; ++s)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[s][i] = v4i{0, 0, 0, 0};

    // codes in LDS: source, group of 16 k, row, 16 bytes
    const int src_bytes = n16w * MT * 256;
#pragma unroll
    for (int s = 0; s < SRC; ++s) {
        if (IN == GNN_I8) {
            if (threadIdx.x < kFewRows) {
                const int r = (int)threadIdx.x < M ? (int)threadIdx.x : M - 1;
                s_row[s][threadIdx.x] = a.sa[s][a.in_rows ? a.in_rows[r] : r];
            }
        } else {
            constexpr int DT = IN == GNN_F32 ? GNN_F32 : GNN_BF16;
            for (int r = wave; r < M; r += 8) {
                const int64_t v = a.in_rows ? (int64_t)a.in_rows[r] : r;
                uint32_t top = 0;
                float x[2][8];
                for (int c0 = lane * 8; c0 < K; c0 += 1024) {     // two groups at once; a row of up to 1024 stays in registers
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        load8<DT, AL>(a.A[s], v * a.lda, c0 + 512 * k, K, x[k]);
                        top = largest_pattern(x[k], top);
                    }
                }
                const RowGrid g = row_grid(wave_max_u32(top));
                for (int c0 = lane * 8; c0 < n16w * 16; c0 += 1024) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int c = c0 + 512 * k;
                        if (c >= n16w * 16) continue;
                        if (K > 1024 || lane * 8 >= K) load8<DT, AL>(a.A[s], v * a.lda, c, K, x[k]);
                        *(uint2*)(lds + s * src_bytes + ((c / 16) * (MT * 16) + r) * 16 + c % 16) = codes_of<DT>(x[k], g);
                    }
                }
                if (lane == 0) s_row[s][r] = g.scale;
            }
        }
    }
    if (IN != GNN_I8) __syncthreads();

#pragma unroll
    for (int s = 0; s < SRC; ++s) {
        const int8_t* w = a.W[s] + (int64_t)(n0 / 32) * n16w * 512 + kg * 512 + (n0 % 32 + col) * 16;
        const int8_t* from[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            if (IN == GNN_I8) {
                const int r = i * 16 + col < M ? i * 16 + col : M - 1;
                from[i] = (const int8_t*)a.A[s] + (a.in_rows ? (int64_t)a.in_rows[r] : r) * a.lda;
            } else {
                from[i] = lds + s * src_bytes + (i * 16 + col) * 16;
            }
        }
        for (int k0 = wave; k0 < steps; k0 += 32) {
            v4i fb[4], fa[4][MT];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const int k = k0 + 8 * d < steps ? k0 + 8 * d : k0;
                fb[d] = *(const v4i*)(w + (int64_t)k * 2048);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (IN == GNN_I8) {
                        const int c = (4 * k + kg) * 16;      // beyond K the weights are zeros
                        fa[d][i] = *(const v4i*)(from[i] + (c < K ? c : 0));
                    } else {
                        fa[d][i] = *(const v4i*)(from[i] + (4 * k + kg) * (MT * 256));
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < 4; ++d)
                if (k0 + 8 * d < steps) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[s][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[d], fa[d][i], acc[s][i], 0, 0, 0);
                }
        }
    }
    __syncthreads();      // the codes are read: the partial sums take their place
    v4i* red = (v4i*)lds;
#pragma unroll
    for (int s = 0; s < SRC; ++s)
#pragma unroll
        for (int i = 0; i < MT; ++i) red[((s * MT + i) * 8 + wave) * 64 + lane] = acc[s][i];
    __syncthreads();
    if (wave >= MT) return;
    const int r = wave * 16 + col, n = n0 + 4 * kg;
    if (r >= M || n >= a.N) return;
    float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < SRC; ++s) {
        v4i t = red[(s * MT + wave) * 8 * 64 + lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) t += red[((s * MT + wave) * 8 + k) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float w = a.sw[s][n + e < a.N ? n + e : 0];
            y[e] += (float)t[e] * (s_row[s][r] * w);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += a.bias ? a.bias[n + e < a.N ? n + e : 0] : 0.f;
    const int64_t v = a.rows ? (int64_t)a.rows[r] : r;
    if (a.out_dtype == GNN_F32) store_four<GNN_F32>(a, v, n, y);
    else store_four<GNN_BF16>(a, v, n, y);
}

template <int IN, int AL>
static int32_t launch_few(const LinearI8& a, hipStream_t stream) {
    const int grid = (a.N + 15) / 16;
    if (a.n_src == 2) {
        if (a.n_active <= 16) linear_i8_few_kernel<IN, AL, 1, true><<<grid, 512, 0, stream>>>(a);
        else linear_i8_few_kernel<IN, AL, 2, true><<<grid, 512, 0, stream>>>(a);
    } else {
        if (a.n_active <= 16) linear_i8_few_kernel<IN, AL, 1, false><<<grid, 512, 0, stream>>>(a);
        else linear_i8_few_kernel<IN, AL, 2, false><<<grid, 512, 0, stream>>>(a);
    }
    GNN_LAUNCH_CHECK("linear_i8_few_kernel");
    return GNN_OK;
}

// us of one source by tile, 4096 -> 4096 unless given (both sides of a line on the same card, before the last 5 to 10 % that all tiles gained):
// 128 rows 13.4 with 64, 22.4 with 128; 300 rows 16.7, 23.2; 1000 rows (256 tiles of 128) 35.8, 27.0, with 256 (64 tiles) 54.2;
// 2000 x 2048 -> 2048 (256 of 128) 20.5, 17.6; 4096 rows (256 of 256) 138, 86, 74; 8192 rows 170 with 128, 142 with 256.
// Now 13.2, 16.2, 25.5, 16.2, 68 and 129 to 132 with the tile taken.
constexpr int kTiles256 = 192, kTiles128 = 256;

template <int OUT>
static int32_t launch_tiles(const LinearI8& a, hipStream_t stream) {
    const auto tiles = [&](int64_t m, int64_t n) { return (a.n_active + m - 1) / m * ((a.N + n - 1) / n); };
    if (a.n_src == 1 && tiles(256, 256) >= kTiles256) return launch_tile<OUT, 4, 2, 2, 4, 4, false>(a, stream);
    if (tiles(128, 128) >= kTiles128) return a.n_src == 2 ? launch_tile<OUT, 2, 2, 2, 2, 4, true>(a, stream) : launch_tile<OUT, 2, 2, 2, 2, 4, false>(a, stream);
    return a.n_src == 2 ? launch_tile<OUT, 1, 1, 2, 2, 4, true>(a, stream) : launch_tile<OUT, 1, 1, 2, 2, 4, false>(a, stream);
}

// How a call runs, by its sizes alone.
enum Route { kFew, kPanel, kTile };

// us by route (MI355X; the tiles before their last gain of 5 to 10 %):
//                             rows x K -> N, sources      panel   tile 128
//   bfloat16, up to 1024 columns  200 000 x 512 -> 512        140     187     (a launch before the tile kernel makes the codes)
//                                 200 000 x 602 -> 256, two   172     315
//                                 3000 x 1024 -> 4096          32      31
//                                 200 x 128 -> 64             4.7     6.3     (float)
//   codes                         200 000 x 602 -> 256, two   130     177
//                                 300 000 x 400 -> 512        165     185
//                                 200 000 x 256 -> 256         52      53
//                                 200 000 x 1024 -> 256       117     103
//                                 1 000 000 x 128 -> 64       155     122
//                                 50 000 x 602 -> 41           21      20
// Not measured on both sides: float rows of up to 1024 columns with outputs wider than 512, other than the 3000 rows above, and 33 to 200 of them
// (fewer than 8 tiles leave dies of the panel kernel's idle).
//   32 rows x 4096 -> 4096: 7.8 with the kernel for few rows, 13 with tiles of 64; 8 rows from bfloat16 9.1 and 16.7.
static Route route_of(int32_t n_active, int32_t K, int32_t N, bool codes) {
    if (n_active <= kFewRows) return kFew;
    if (codes) return K <= 640 && N > 64 ? kPanel : kTile;
    return K <= 1024 ? kPanel : kTile;
}

// Whether the kernel of that route puts float rows on the grid itself; if not, a launch before it does.
static bool codes_inside(Route r, int32_t n_active, int32_t K, int32_t n_src) {
    if (r == kFew) return (int64_t)((K + 63) / 64 * 64) * (n_active <= 16 ? 16 : 32) * n_src <= kFewCodes;
    return r == kPanel;
}

template <int IN, int AL>
static int32_t launch_with(Route r, const LinearI8& a, hipStream_t stream) {
    if (r == kFew) return launch_few<IN, AL>(a, stream);
    return launch_panel<IN, AL>(a, stream);
}

static int32_t launch_product(Route r, const LinearI8& a, int32_t in_dtype, hipStream_t stream) {
    if (r == kTile) return a.out_dtype == GNN_F32 ? launch_tiles<GNN_F32>(a, stream) : launch_tiles<GNN_BF16>(a, stream);
    if (in_dtype == GNN_I8) return launch_with<GNN_I8, 16>(r, a, stream);
    int al = 16;
    for (int k = 0; k < a.n_src; ++k) {
        const int own = in_dtype == GNN_F32 ? row_alignment<GNN_F32>(a.A[k], a.lda) : row_alignment<GNN_BF16>(a.A[k], a.lda);
        al = own < al ? own : al;
    }
    // rows that do not all start on 16 bytes are read element by element
    if (in_dtype == GNN_F32) return al == 16 ? launch_with<GNN_F32, 16>(r, a, stream) : launch_with<GNN_F32, 4>(r, a, stream);
    return al == 16 ? launch_with<GNN_BF16, 16>(r, a, stream) : launch_with<GNN_BF16, 2>(r, a, stream);
}

}  // namespace gnnhot

using namespace gnnhot;

extern "C" int32_t gnn_linear_i8_fwd(const int32_t* rows, int32_t n_active, const void* A_neigh, const float* scale_neigh, const void* X_self,
                                     const float* scale_self, int64_t ld_in, int32_t K, int32_t in_dtype, const int8_t* Wq_neigh,
                                     const float* wscale_neigh, const int8_t* Wq_self, const float* wscale_self, const float* bias, int32_t N,
                                     void* H_out, int64_t ld_out, int32_t relu, int32_t out_dtype, void* ws, size_t* ws_bytes, void* stream_) {
    hipStream_t stream = (hipStream_t)stream_;
    GNN_REQUIRE(n_active >= 0, GNN_ERR_INVALID_ARG, "negative row count");
    GNN_REQUIRE(in_dtype == GNN_I8 || in_dtype == GNN_F32 || in_dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "unknown input dtype %d", in_dtype);
    GNN_REQUIRE(out_dtype == GNN_F32 || out_dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "unknown output dtype %d", out_dtype);
    GNN_REQUIRE(K >= 1 && N >= 1, GNN_ERR_INVALID_ARG, "K = %d, N = %d", K, N);
    GNN_REQUIRE(K <= kMaxI8K && N <= kMaxI8N, GNN_ERR_UNSUPPORTED, "K = %d, N = %d are over %d, %d", K, N, kMaxI8K, kMaxI8N);
    GNN_REQUIRE(ld_in >= K && ld_out >= N, GNN_ERR_SHAPE, "leading dimension smaller than the width");
    const bool codes = in_dtype == GNN_I8;
    GNN_REQUIRE(!codes || (ld_in % 16 == 0), GNN_ERR_SHAPE, "ld_in = %lld: rows of codes start on 16 bytes", (long long)ld_in);
    GNN_REQUIRE((X_self == nullptr) == (Wq_self == nullptr), GNN_ERR_INVALID_ARG, "X_self and Wq_self go together");
    const int n_src = Wq_self ? 2 : 1;
    const int64_t Kq = (K + 15) / 16 * 16;
    const Route route = route_of(n_active, K, N, codes);
    const bool before = !codes && !codes_inside(route, n_active, K, n_src);    // the rows' codes are made in ws first
    WsCarver carve(ws);
    int8_t* q[2] = {nullptr, nullptr};
    float* s[2] = {nullptr, nullptr};
    if (before)
        for (int k = 0; k < n_src; ++k) {
            q[k] = carve.take<int8_t>((size_t)(n_active * Kq));
            s[k] = carve.take<float>((size_t)n_active);
        }
    bool query;
    GNN_CHECK(ws_protocol(ws, ws_bytes, carve.used, &query));
    if (query) return GNN_OK;
    if (n_active == 0) return GNN_OK;
    GNN_REQUIRE(A_neigh != nullptr && Wq_neigh != nullptr && wscale_neigh != nullptr && H_out != nullptr, GNN_ERR_INVALID_ARG, "NULL argument");
    GNN_REQUIRE(n_src == 1 || wscale_self != nullptr, GNN_ERR_INVALID_ARG, "wscale_self is NULL");
    GNN_REQUIRE(!codes || (scale_neigh != nullptr && (n_src == 1 || scale_self != nullptr)), GNN_ERR_INVALID_ARG, "codes without scales");
    GNN_REQUIRE((((uintptr_t)Wq_neigh | (uintptr_t)Wq_self) & 15u) == 0, GNN_ERR_INVALID_ARG, "packed weights are not 16-byte aligned");
    GNN_REQUIRE(!codes || (((uintptr_t)A_neigh | (uintptr_t)X_self) & 15u) == 0, GNN_ERR_INVALID_ARG, "codes are not 16-byte aligned");
    LinearI8 a = {};
    a.rows = rows;
    a.n_active = n_active;
    a.K = K;
    a.W[0] = Wq_neigh;
    a.W[1] = Wq_self;
    a.sw[0] = wscale_neigh;
    a.sw[1] = wscale_self;
    a.bias = bias;
    a.N = N;
    a.H = H_out;
    a.ldh = ld_out;
    a.relu = relu;
    a.n_src = n_src;
    const int es = out_dtype == GNN_F32 ? 4 : 2;
    a.vec_out = ((uintptr_t)H_out % (4 * es)) == 0 && ld_out % 4 == 0;
    a.vec_out8 = ((uintptr_t)H_out % (8 * es)) == 0 && ld_out % 8 == 0;
    a.out_dtype = out_dtype;
    a.in_rows = rows;
    a.lda = ld_in;
    a.A[0] = A_neigh;
    a.A[1] = X_self;
    a.sa[0] = scale_neigh;
    a.sa[1] = scale_self;
    if (before) {
        for (int k = 0; k < n_src; ++k) {
            const QuantRows r = {rows, n_active, a.A[k], ld_in, K, q[k], Kq, s[k], nullptr, 0, true};
            GNN_CHECK(quantize_rows(r, in_dtype, stream));
            a.A[k] = q[k];
            a.sa[k] = s[k];
        }
        a.in_rows = nullptr;
        a.lda = Kq;
    }
    return launch_product(route, a, before ? (int32_t)GNN_I8 : in_dtype, stream);
}
