// What a training program does with its gradients: their norm (two launches), and the AdamW step on every tensor of a model (one).
//
// Both calls walk a table of tensors (gnn_param) that lies in device memory.  A tensor is cut into chunks of kChunk
// elements, the chunks of all tensors are numbered through, and a workgroup takes a run of them: it finds the tensor of its
// first chunk by a 64-way search over the tensors' first chunks (one load a level, two levels up to 4096 tensors) and walks
// forward from there, so a model of hundreds of small tensors costs the same launch as one large one.
#include "common.h"

#include <math.h>

namespace gnnhot {

// The codes of an 8-bit state are defined by their operations in 32 bits, each rounded on its own.
#pragma clang fp contract(off)

constexpr int kChunk = 1024;       // elements of a chunk; a multiple of the state block
constexpr int kStateBlock = 256;   // elements of an 8-bit state that share a scale: one wavefront of four each
constexpr int kMaxGrid = 2048;

// The tensor of a chunk: the last one whose first chunk is not beyond it (empty tensors share theirs with the next and are never the last).
__device__ __forceinline__ int find_tensor(const gnn_param* __restrict__ t, int n, int64_t chunk) {
    int lo = 0, cnt = n;   // uniform over the wavefront
    while (cnt > 1) {
        const int stride = (cnt + 63) / 64;
        const int j = lane_id() * stride;
        const bool below = j < cnt && t[lo + j].first_chunk <= chunk;
        const int last = __popcll(__ballot(below)) - 1;    // first chunks ascend: the lanes below are a prefix
        lo += last * stride;
        cnt = cnt - last * stride < stride ? cnt - last * stride : stride;
    }
    return lo;
}

template <int DT, bool VEC>
__device__ __forceinline__ void load4(const void* p, int64_t i, int64_t n, float (&x)[4]) {
    if (VEC) {
        if (DT == GNN_F32) {
            const float4 r = *(const float4*)((const float*)p + i);
            x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
        } else {
            const uint2 r = *(const uint2*)((const uint16_t*)p + i);
            x[0] = bf16lo(r.x); x[1] = bf16hi(r.x); x[2] = bf16lo(r.y); x[3] = bf16hi(r.y);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = 0.f;
            if (i + e < n) x[e] = DT == GNN_F32 ? ((const float*)p)[i + e] : bf16_to_f32(((const uint16_t*)p)[i + e]);
        }
    }
}

template <int DT, bool VEC>
__device__ __forceinline__ void store4(void* p, int64_t i, int64_t n, const float (&x)[4]) {
    if (VEC) {
        if (DT == GNN_F32) *(float4*)((float*)p + i) = make_float4(x[0], x[1], x[2], x[3]);
        else *(uint2*)((uint16_t*)p + i) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) {
                if (DT == GNN_F32) ((float*)p)[i + e] = x[e];
                else ((uint16_t*)p)[i + e] = f32_to_bf16(x[e]);
            }
    }
}

template <bool VEC>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t i, int64_t n) {
    if (VEC) return *(const uint32_t*)(p + i);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n) w |= (uint32_t)p[i + e] << (8 * e);
    return w;
}

template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int64_t n, uint32_t w) {
    if (VEC) {
        *(uint32_t*)(p + i) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i + e < n) p[i + e] = (uint8_t)(w >> (8 * e));
    }
}

// ---- norm of all gradients ---------------------------------------------------------------------------------------
// Sum of squares in 64 bits: a square of a float is exact there, so the sum is good to about n 2^-53 whatever its order and
// its 32-bit root does not depend on the split.  Bound: HBM, one read of the gradients (the 64-bit multiply-adds are a
// twentieth of what the bytes take).  59M floats in 558 tensors 36 us in a loop of its own (6.5 TB/s, part of it from the last-level cache, which
// holds 256 MB), 78 us after a step that moved 942 MB (3.0 TB/s); 247M 213 us after a step (4.6 TB/s); 0.46M 3.3 us.
template <int DT, bool VEC>
__device__ __forceinline__ double square_range(const void* g, int64_t i0, int64_t i1) {
    double s = 0.0;
    int64_t w = i0 + 4 * (int64_t)(threadIdx.x & ~63u);   // of the wavefront
    const int64_t off = 4 * lane_id();
    if (VEC) {
        for (; w + 3 * 1024 + 256 <= i1; w += 4 * 1024) {   // four loads on their way
            float x[4][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) load4<DT, true>(g, w + 1024 * k + off, i1, x[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fma((double)x[k][e], (double)x[k][e], s);
        }
    }
    for (; w < i1; w += 1024) {
        float x[4];
        if (VEC && w + 256 <= i1) load4<DT, true>(g, w + off, i1, x);
        else load4<DT, false>(g, w + off, i1, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma((double)x[e], (double)x[e], s);
    }
    return s;
}

__device__ __forceinline__ double block_sum(double s, double* lds) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, kWave);
    if (lane_id() == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const gnn_param* __restrict__ params, int32_t n_params, int64_t n_chunks,
                                                        double* __restrict__ part) {
    __shared__ double lds[4];
    const int64_t per = (n_chunks + gridDim.x - 1) / gridDim.x;
    const int64_t c0 = (int64_t)blockIdx.x * per, c1 = c0 + per < n_chunks ? c0 + per : n_chunks;
    double s = 0.0;
    if (c0 < c1) {
        int t = find_tensor(params, n_params, c0);
        for (int64_t c = c0; c < c1 && t < n_params; ++t) {   // uniform over the workgroup
            const void* g = params[t].grad;
            const int64_t n = params[t].n, first = params[t].first_chunk;
            const int dt = params[t].grad_dtype;
            const int64_t after = first + (n + kChunk - 1) / kChunk, stop = after < c1 ? after : c1;
            const int64_t i0 = (c - first) * kChunk, end = (stop - first) * kChunk, i1 = end < n ? end : n;
            const bool vec = ((uintptr_t)g & (dt == GNN_F32 ? 15u : 7u)) == 0;
            if (dt == GNN_F32) s += vec ? square_range<GNN_F32, true>(g, i0, i1) : square_range<GNN_F32, false>(g, i0, i1);
            else s += vec ? square_range<GNN_BF16, true>(g, i0, i1) : square_range<GNN_BF16, false>(g, i0, i1);
            c = stop;
        }
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// A launch of its own: a count of finished workgroups in device memory (one launch) costs 28 ns for each of them, one after the other -
// 58 us for the 1960 workgroups of a model of 59 MB, where the sum itself takes 15.  A model of 452 chunks was faster with the count: the two
// kernels took 6.5 us together and take 9 with this launch (2 us and the gap); a line between the two forms was not measured.
__global__ __launch_bounds__(256) void norm_state_kernel(const double* __restrict__ part, int32_t n_part, float grad_scale, float max_norm,
                                                         gnn_step_state* __restrict__ state) {
    __shared__ double lds[4];
    double total = 0.0;
#pragma unroll
    for (int k = 0; k < kMaxGrid / 256; ++k) {    // all loads at once
        const int i = k * 256 + (int)threadIdx.x;
        total += i < n_part ? part[i] : 0.0;
    }
    total = block_sum(total, lds);
    if (threadIdx.x != 0) return;
    const double norm = fabs((double)grad_scale) * sqrt(total);
    const bool ok = isfinite((float)norm);     // as it is stored: finite gradients whose norm is no float are refused too
    state->ok = ok;
    state->sum_sq = total;
    state->norm = (float)norm;
    state->coef = (float)((double)grad_scale * (max_norm > 0.f && norm > (double)max_norm ? (double)max_norm / norm : 1.0));
    if (ok) state->step += 1;
    else state->skipped += 1;
}

// ---- AdamW ---------------------------------------------------------------------------------------------------------
struct AdamArgs {
    float b1, ob1, b2, ob2, eps;    // ob = 1 - b
    float grad_scale, step_size, inv_root;   // without a state: lr / (1 - b1^t), 1 / sqrt(1 - b2^t) from the host
    double lr, beta1, beta2;
    int64_t step;        // without a state
    uint32_t seed;       // of the unbiased rounding
};

// eps is what divides the update where a second moment in float is too small to: the square of a gradient below 2^-75 is no float, and a
// block of 8-bit moments ends at 2^-126, whose root, corrected for beta2 = 0.999's first step, is 3.4e-18.  With an eps below that the step of
// such a weight would be m / eps, larger without bound than the formula's; below 2.9e-39 even 1 / eps is infinite, and a weight
// that nothing has reached (m = 0) would become NaN.  The upper end keeps the reciprocal a normal float.
constexpr float kEpsLeast = 1e-16f, kEpsMost = 1e30f;

// beta^t by squaring; t is the same for every lane
__device__ __forceinline__ double power(double b, int64_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return r;
}

// 8-bit states.  First moment: m = scale f |f|, f = c / 127.  Second moment: v = scale f^4, f = c / 255.  The steps of m are finest near
// zero, those of v are about even in its logarithm over nine decades, where a linear code would lose all but the block's largest.
__device__ __forceinline__ float m_value(int c, float scale) {
    const float f = (float)c * (1.0f / 127.0f);
    return scale * (f * fabsf(f));
}
__device__ __forceinline__ float v_value(int c, float scale) {
    float f = (float)c * (1.0f / 255.0f);
    f = f * f;
    return scale * (f * f);
}
// The code of a share x of the scale = the number of borders ((j + 1/2) / 127)^2 at or below x (power 4 and 255 for v).  The root, good to
// an ulp or two, is at most one off next to a border; the borders on its two sides decide.  No border is at or below zero, and the one
// above the last code is above 1 by more than x can be.  Without branches: with them the code took a third of the kernel's instructions.
__device__ __forceinline__ float m_code(float x) {
    const float c = floorf(__builtin_amdgcn_sqrtf(x) * 127.0f + 0.5f);
    const float lo = fmaxf(c - 0.5f, 0.f) * (1.0f / 127.0f), hi = (c + 0.5f) * (1.0f / 127.0f);
    return c + (x >= hi * hi ? 1.0f : 0.f) - (x < lo * lo ? 1.0f : 0.f);
}
__device__ __forceinline__ float v_code(float x) {
    const float c = floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(x)) * 255.0f + 0.5f);
    float lo = fmaxf(c - 0.5f, 0.f) * (1.0f / 255.0f), hi = (c + 0.5f) * (1.0f / 255.0f);
    lo = lo * lo;
    hi = hi * hi;
    return c + (x >= hi * hi ? 1.0f : 0.f) - (x < lo * lo ? 1.0f : 0.f);
}

// Unbiased rounding.  To the nearest code a state that moves by less than half a step of its code never moves: a second moment falls by at
// most 1 - beta2 of itself a step, a code is 4 / c of it, so none but the block's largest ever falls, and it rises on spikes only.
// Gradients of N(0, 1), 64 of a block's 256 falling tenfold after 1000 steps: their second moments are 70 times the 32-bit ones 6000
// steps later, their steps eight times too small.  Here x between the values of codes c and c + 1 becomes c + 1 in as many of 2^23 cases as x
// lies beyond c's value, so that its mean is x: the same second moments are within 0.7 to 1.4 of the 32-bit ones (a relative spread of
// about sqrt(2 / c)) and a first moment whose gradient has become zero decays to zero.
// The draw is a function of (seed, step, tensor, element) alone: products of 32 bits by odd constants (the fractions of the golden ratio and of
// the roots of 3 and 2), their halves folded onto each other; m takes the upper 23 bits of the element's number, v the lower 23 in
// reverse.  Uniform and without correlation between elements, steps, tensors and the two (1M draws in 4096 cells each).
// What it costs: four products a draw at a quarter of the vector unit's rate, which the step is close to being bound by: 247M elements 889 to 914 us
// (819 with nearest codes), 59M 239 to 260 (183 to 207).
constexpr uint32_t kDraw[3] = {0x9E3779B9u, 0xBB67AE85u, 0x6A09E667u};
__device__ __forceinline__ uint32_t fold(uint32_t x, uint32_t c) {
    const uint64_t p = (uint64_t)x * c;
    return (uint32_t)p ^ (uint32_t)(p >> 32);
}
struct DrawKey {      // of a tensor in a step
    uint32_t k0, k1;
};
__device__ __forceinline__ DrawKey draw_key(uint32_t seed, int64_t step, uint32_t tensor) {
    uint32_t s = fold(seed + kDraw[0], kDraw[1]);
    s = fold(s ^ (uint32_t)step, kDraw[2]);
    s = fold(s + (uint32_t)(step >> 32) + kDraw[0], kDraw[1]);
    const uint32_t k0 = fold(s ^ tensor, kDraw[2]);
    return {k0, fold(k0 + kDraw[0], kDraw[1])};
}
// Of the elements from i on that share its upper 32 bits (four, and i a multiple of four).
__device__ __forceinline__ DrawKey key_at(const DrawKey& k, int64_t i) {
    const uint32_t high = (uint32_t)(i >> 32);
    return {k.k0 + high * kDraw[2], k.k1 + high * kDraw[0]};
}
__device__ __forceinline__ uint32_t draw(const DrawKey& k, uint32_t low) { return fold(fold(low ^ k.k0, kDraw[0]) ^ k.k1, kDraw[1]); }
// (k + 1/2) 2^-23 of the upper 23 bits k, exact
__device__ __forceinline__ float unit(uint32_t h) { return __uint_as_float(0x3f800000u | h >> 9) - 0.99999994f; }

// POWER 2 and 127 steps, or 4 and 255: the number of values (j / steps)^POWER at or below x, j from 1 on, and one more where
// x - (that value) > u * (the distance to the next value).  x may be an ulp above 1.
template <int POWER>
__device__ __forceinline__ float unbiased_code(float x, float u) {
    constexpr float kSteps = POWER == 2 ? 127.0f : 255.0f;
    const auto value = [](float c) {
        float f = c * (1.0f / kSteps);
        f = f * f;
        return POWER == 2 ? f : f * f;
    };
    float r = __builtin_amdgcn_sqrtf(x);
    if (POWER == 4) r = __builtin_amdgcn_sqrtf(r);
    float c = floorf(r * kSteps);                 // at most one off: the values on its two sides decide
    c = c + (x >= value(c + 1.0f) ? 1.0f : 0.f) - (x < value(c) ? 1.0f : 0.f);
    const float lo = value(c), hi = value(c + 1.0f);
    return fminf(c + (x - lo > u * (hi - lo) ? 1.0f : 0.f), kSteps);
}

// A scale from the largest bit pattern of |x| in a block: bit patterns of non-negative floats ascend with their values, infinities and NaN
// last.  A block that holds one of those gets the scale NaN (all its values are NaN from then on: nothing is hidden), one below the
// smallest normal float becomes zeros.
__device__ __forceinline__ float scale_of(uint32_t top) {
    if (top >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    return top < 0x00800000u ? 0.f : __uint_as_float(top);
}

// Root of the instruction set, good to an ulp.  It takes a subnormal for zero: a lane that has one (a pattern of 1 .. 2^23 - 1) takes its
// four roots again, 2^64 times as large, so that 2^-126 and the values below it divide as the formula says.  Ordinary
// values pay for the question alone.
__device__ __forceinline__ void roots(const float (&v)[4], float (&r)[4]) {
    uint32_t least = 0xffffffffu;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t b = __float_as_uint(v[e]) - 1u;      // of zero: the largest
        least = b < least ? b : least;
        r[e] = __builtin_amdgcn_sqrtf(v[e]);
    }
    if (least < 0x007fffffu) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (__float_as_uint(v[e]) < 0x00800000u) r[e] = __builtin_amdgcn_sqrtf(v[e] * 0x1p64f) * 0x1p-32f;
    }
}

// A wavefront takes 256 elements at a time, four a lane: 16-byte loads and stores of floats, and exactly one block of an 8-bit state, whose
// largest value is then a reduction inside the wavefront.  Bound: HBM.  28 bytes an element with float states, 16 with 8-bit states:
// 247M elements in 8 bits, nearest codes, 819 us (4.8 TB/s, the rate of a copy of 4 GB; the vector unit is busy for 84 %), 59M 183 to 207 us, 0.46M with float states 5.4 us.
// With the codes found by IEEE roots and branches the 8-bit form was bound by the vector unit instead: 938 and 261 us.
struct AdamTensor {
    void* param;
    const void* grad;
    void* m;
    void* v;
    float *m_scale, *v_scale, *master;
    int64_t n;
    float decay;   // 1 - lr weight_decay
};

// PT: 0 float parameters, 1 bfloat16, 2 bfloat16 with a float copy that is updated and rounded into them.
template <int PT, int GT, int BITS, bool UNBIASED, bool VEC>
__device__ __forceinline__ void adamw_four(const AdamTensor& t, int64_t i, const AdamArgs& a, float coef, float step_size, float inv_root,
                                           const DrawKey& key) {
    float p[4], g[4], m[4], v[4];
    const int64_t n = t.n;
    uint32_t mc = 0, vc = 0;
    float ms = 0.f, vs = 0.f;
    load4<PT == 1 ? GNN_BF16 : GNN_F32, VEC>(PT == 2 ? (const void*)t.master : t.param, i, n, p);
    load4<GT, VEC>(t.grad, i, n, g);
    const int64_t block = i / kStateBlock;   // the same for the whole wavefront
    if (BITS == 32) {
        load4<GNN_F32, VEC>(t.m, i, n, m);
        load4<GNN_F32, VEC>(t.v, i, n, v);
    } else {
        mc = load_codes<VEC>((const uint8_t*)t.m, i, n);
        vc = load_codes<VEC>((const uint8_t*)t.v, i, n);
        ms = t.m_scale[block];
        vs = t.v_scale[block];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = m_value((int8_t)(mc >> (8 * e)), ms);
            v[e] = v_value((int)((vc >> (8 * e)) & 255u), vs);
        }
    }
    uint32_t mt = 0, vt = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float gs = g[e] * coef;
        m[e] = m[e] * a.b1 + gs * a.ob1;
        v[e] = v[e] * a.b2 + (gs * gs) * a.ob2;
    }
    float root[4];
    roots(v, root);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float den = root[e] * inv_root + a.eps;      // at least kEpsLeast
        p[e] = p[e] * t.decay - (m[e] * __builtin_amdgcn_rcpf(den)) * step_size;
        if (BITS == 8 && (VEC || i + e < n)) {
            const uint32_t x = __float_as_uint(m[e]) & 0x7fffffffu, y = __float_as_uint(v[e]) & 0x7fffffffu;
            mt = x > mt ? x : mt;
            vt = y > vt ? y : vt;
        }
    }
    if (PT == 2) store4<GNN_F32, VEC>(t.master, i, n, p);
    store4<PT == 0 ? GNN_F32 : GNN_BF16, VEC>(t.param, i, n, p);
    if (BITS == 32) {
        store4<GNN_F32, VEC>(t.m, i, n, m);
        store4<GNN_F32, VEC>(t.v, i, n, v);
    } else {
        ms = scale_of(wave_max_u32(mt));
        vs = scale_of(wave_max_u32(vt));
        const float mi = ms > 0.f ? 1.0f / ms : 0.f, vi = vs > 0.f ? 1.0f / vs : 0.f;   // zeros and NaN: codes 0
        mc = vc = 0;
        const DrawKey at = key_at(key, i);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t h = UNBIASED ? draw(at, (uint32_t)i + e) : 0u;
            float c = UNBIASED ? unbiased_code<2>(fabsf(m[e]) * mi, unit(h)) : m_code(fabsf(m[e]) * mi);
            c = mi > 0.f ? c : 0.f;
            c = m[e] < 0.f ? -c : c;
            float d = UNBIASED ? unbiased_code<4>(v[e] * vi, unit(__brev(h))) : v_code(v[e] * vi);
            d = v[e] > 0.f ? fmaxf(d, 1.0f) : 0.f;     // a second moment never shrinks to zero: its root divides
            d = vi > 0.f ? d : 0.f;
            mc |= ((uint32_t)(int)c & 255u) << (8 * e);
            vc |= (uint32_t)d << (8 * e);
        }
        store_codes<VEC>((uint8_t*)t.m, i, n, mc);
        store_codes<VEC>((uint8_t*)t.v, i, n, vc);
        if (lane_id() == 0) {
            t.m_scale[block] = ms;
            t.v_scale[block] = vs;
        }
    }
}

template <int PT, int GT, int BITS, bool UNBIASED>
__device__ __forceinline__ void adamw_chunks(const AdamTensor& t, int64_t i0, int64_t i1, bool vec, const AdamArgs& a, float coef,
                                             float step_size, float inv_root, const DrawKey& key) {
    // a wavefront owns whole state blocks; it enters a block together, also where the tensor ends inside it
    for (int64_t w = i0 + (threadIdx.x & ~63u) * 4; w < i1; w += 1024) {
        const int64_t i = w + 4 * lane_id();
        if (vec && w + kStateBlock <= t.n) adamw_four<PT, GT, BITS, UNBIASED, true>(t, i, a, coef, step_size, inv_root, key);
        else adamw_four<PT, GT, BITS, UNBIASED, false>(t, i, a, coef, step_size, inv_root, key);
    }
}

template <bool UNBIASED>
__global__ __launch_bounds__(256) void adamw_kernel(const gnn_param* __restrict__ params, int32_t n_params, int64_t n_chunks, AdamArgs a,
                                                    const float* __restrict__ lr_device, const gnn_step_state* __restrict__ state) {
    const int64_t per = (n_chunks + gridDim.x - 1) / gridDim.x;
    const int64_t c0 = (int64_t)blockIdx.x * per, c1 = c0 + per < n_chunks ? c0 + per : n_chunks;
    if (c0 >= c1) return;
    double lr = a.lr;
    if (lr_device) lr = (double)*lr_device;
    float coef = a.grad_scale, step_size = a.step_size, inv_root = a.inv_root;
    int64_t step = a.step;
    if (state) {
        if (!state->ok) return;   // a refused step changes nothing
        coef = state->coef;
        step = state->step;
        step_size = (float)(lr / (1.0 - power(a.beta1, step)));
        inv_root = (float)(1.0 / sqrt(1.0 - power(a.beta2, step)));
    } else if (lr_device) {
        step_size = (float)(lr * (double)a.step_size);
    }
    int k = find_tensor(params, n_params, c0);
    for (int64_t c = c0; c < c1 && k < n_params; ++k) {   // uniform over the workgroup
        const gnn_param& q = params[k];
        const int64_t first = q.first_chunk, after = first + (q.n + kChunk - 1) / kChunk;
        const int64_t stop = after < c1 ? after : c1;
        const int bits = q.state_bits, gt = q.grad_dtype, pt = q.param_dtype == GNN_F32 ? 0 : q.master ? 2 : 1;
        if (bits != 0 && c < stop) {
            const AdamTensor t = {q.param, q.grad, q.m, q.v, q.m_scale, q.v_scale, q.master, q.n, (float)(1.0 - lr * (double)q.weight_decay)};
            // vectors of four: 16 bytes of a float, 8 of a bfloat16, 4 of an 8-bit array
            const uintptr_t off = ((uintptr_t)q.param & (pt ? 7u : 15u)) | ((uintptr_t)q.grad & (gt == GNN_F32 ? 15u : 7u)) |
                                  (((uintptr_t)q.m | (uintptr_t)q.v) & (bits == 32 ? 15u : 3u)) | ((uintptr_t)q.master & 15u);
            const bool vec = off == 0;
            const DrawKey key = UNBIASED ? draw_key(a.seed, step, (uint32_t)k) : DrawKey{0u, 0u};
            const int64_t i0 = (c - first) * kChunk, end = (stop - first) * kChunk, i1 = end < q.n ? end : q.n;
#define GNN_ADAM(PT_, GT_, B_) adamw_chunks<PT_, GT_, B_, B_ == 8 && UNBIASED>(t, i0, i1, vec, a, coef, step_size, inv_root, key)
#define GNN_ADAM_P(GT_, B_)                 \
    do {                                    \
        if (pt == 0) GNN_ADAM(0, GT_, B_);  \
        else if (pt == 1) GNN_ADAM(1, GT_, B_); \
        else GNN_ADAM(2, GT_, B_);          \
    } while (0)
            if (bits == 32) {
                if (gt == GNN_F32) GNN_ADAM_P(GNN_F32, 32);
                else GNN_ADAM_P(GNN_BF16, 32);
            } else {
                if (gt == GNN_F32) GNN_ADAM_P(GNN_F32, 8);
                else GNN_ADAM_P(GNN_BF16, 8);
            }
#undef GNN_ADAM_P
#undef GNN_ADAM
        }
        c = c < stop ? stop : c;
    }
}

// ---- the values an 8-bit state stands for (checkpoints) ---------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(256) void state_values_kernel(const int8_t* __restrict__ m, const float* __restrict__ m_scale,
                                                           const uint8_t* __restrict__ v, const float* __restrict__ v_scale, int64_t n,
                                                           void* __restrict__ m_out, void* __restrict__ v_out, bool vec) {
    for (int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x); i < n; i += 4 * 256 * (int64_t)gridDim.x) {
        const bool whole = vec && i + 4 <= n;
        const uint32_t mc = whole ? load_codes<true>((const uint8_t*)m, i, n) : load_codes<false>((const uint8_t*)m, i, n);
        const uint32_t vc = whole ? load_codes<true>(v, i, n) : load_codes<false>(v, i, n);
        const float ms = m_scale[i / kStateBlock], vs = v_scale[i / kStateBlock];
        float x[4], y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = m_value((int8_t)(mc >> (8 * e)), ms);
            y[e] = v_value((int)((vc >> (8 * e)) & 255u), vs);
        }
        if (whole) {
            store4<DT, true>(m_out, i, n, x);
            store4<DT, true>(v_out, i, n, y);
        } else {
            store4<DT, false>(m_out, i, n, x);
            store4<DT, false>(v_out, i, n, y);
        }
    }
}

static int32_t check_table(const gnn_param* params, int32_t n_params, int64_t n_chunks) {
    GNN_REQUIRE(n_params >= 0 && n_chunks >= 0, GNN_ERR_INVALID_ARG, "negative size");
    GNN_REQUIRE(n_chunks < ((int64_t)1 << 40), GNN_ERR_UNSUPPORTED, "%lld chunks are too many", (long long)n_chunks);
    GNN_REQUIRE(n_chunks == 0 || (params != nullptr && n_params > 0), GNN_ERR_INVALID_ARG, "%lld chunks and no tensors", (long long)n_chunks);
    GNN_REQUIRE(((uintptr_t)params & 7u) == 0, GNN_ERR_INVALID_ARG, "params is not 8-byte aligned");
    return GNN_OK;
}

static int grid_of(int64_t n_chunks) { return (int)(n_chunks < kMaxGrid ? (n_chunks > 0 ? n_chunks : 1) : kMaxGrid); }

}  // namespace gnnhot

using namespace gnnhot;

extern "C" int32_t gnn_param_layout(gnn_param* params_host, int32_t n_params, int64_t* n_chunks_host) {
    GNN_REQUIRE(n_params >= 0, GNN_ERR_INVALID_ARG, "n_params < 0");
    GNN_REQUIRE(n_chunks_host != nullptr && (params_host != nullptr || n_params == 0), GNN_ERR_INVALID_ARG, "NULL argument");
    int64_t chunks = 0;
    for (int32_t i = 0; i < n_params; ++i) {
        gnn_param& p = params_host[i];
        GNN_REQUIRE(p.n >= 0 && p.n < ((int64_t)1 << 48), GNN_ERR_INVALID_ARG, "tensor %d: %lld elements", i, (long long)p.n);
        GNN_REQUIRE(p.grad_dtype == GNN_F32 || p.grad_dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "tensor %d: unknown gradient dtype %d", i, p.grad_dtype);
        GNN_REQUIRE(p.state_bits == 0 || p.state_bits == 8 || p.state_bits == 32, GNN_ERR_UNSUPPORTED, "tensor %d: states of %d bits", i, p.state_bits);
        GNN_REQUIRE(p.grad != nullptr || p.n == 0, GNN_ERR_INVALID_ARG, "tensor %d: grad is NULL", i);
        GNN_REQUIRE(((uintptr_t)p.grad & (p.grad_dtype == GNN_F32 ? 3u : 1u)) == 0, GNN_ERR_INVALID_ARG, "tensor %d: grad is not aligned to its elements", i);
        if (p.state_bits != 0) {
            GNN_REQUIRE(p.param_dtype == GNN_F32 || p.param_dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "tensor %d: unknown parameter dtype %d", i, p.param_dtype);
            GNN_REQUIRE((p.param != nullptr && p.m != nullptr && p.v != nullptr) || p.n == 0, GNN_ERR_INVALID_ARG, "tensor %d: param, m or v is NULL", i);
            GNN_REQUIRE(p.state_bits == 32 || p.n == 0 || (p.m_scale != nullptr && p.v_scale != nullptr), GNN_ERR_INVALID_ARG, "tensor %d: 8-bit states without scales", i);
            GNN_REQUIRE(p.master == nullptr || p.param_dtype == GNN_BF16, GNN_ERR_INVALID_ARG, "tensor %d: a float copy of float parameters", i);
            const uintptr_t four = (p.param_dtype == GNN_F32 ? (uintptr_t)p.param : 0) | (uintptr_t)p.master | (uintptr_t)p.m_scale | (uintptr_t)p.v_scale |
                                   (p.state_bits == 32 ? (uintptr_t)p.m | (uintptr_t)p.v : 0);
            GNN_REQUIRE((four & 3u) == 0 && ((uintptr_t)p.param & 1u) == 0, GNN_ERR_INVALID_ARG, "tensor %d: an array is not aligned to its elements", i);
            GNN_REQUIRE(isfinite(p.weight_decay), GNN_ERR_INVALID_ARG, "tensor %d: weight_decay is not finite", i);
        }
        p.first_chunk = chunks;
        chunks += (p.n + kChunk - 1) / kChunk;
        GNN_REQUIRE(chunks < ((int64_t)1 << 40), GNN_ERR_UNSUPPORTED, "too many elements");
    }
    *n_chunks_host = chunks;
    return GNN_OK;
}

extern "C" int32_t gnn_grad_norm(const gnn_param* params, int32_t n_params, int64_t n_chunks, float grad_scale, float max_norm,
                                 gnn_step_state* state, void* ws, size_t* ws_bytes, void* stream) {
    GNN_CHECK(check_table(params, n_params, n_chunks));
    GNN_REQUIRE(isfinite(grad_scale) && !isnan(max_norm), GNN_ERR_INVALID_ARG, "grad_scale is not finite or max_norm is NaN");
    const int grid = grid_of(n_chunks);
    WsCarver carve(ws);
    double* part = carve.take<double>((size_t)grid);
    bool query;
    GNN_CHECK(ws_protocol(ws, ws_bytes, carve.used, &query));
    if (query) return GNN_OK;
    GNN_REQUIRE(state != nullptr && ((uintptr_t)state & 7u) == 0, GNN_ERR_INVALID_ARG, "state is NULL or not 8-byte aligned");
    grad_norm_kernel<<<grid, 256, 0, (hipStream_t)stream>>>(params, n_params, n_chunks, part);
    GNN_LAUNCH_CHECK("grad_norm_kernel");
    norm_state_kernel<<<1, 256, 0, (hipStream_t)stream>>>(part, grid, grad_scale, max_norm, state);
    GNN_LAUNCH_CHECK("norm_state_kernel");
    return GNN_OK;
}

extern "C" int32_t gnn_adamw_step(const gnn_param* params, int32_t n_params, int64_t n_chunks, const gnn_adamw_hyper* hyper,
                                  const float* lr_device, const gnn_step_state* state, void* stream) {
    GNN_CHECK(check_table(params, n_params, n_chunks));
    GNN_REQUIRE(hyper != nullptr, GNN_ERR_INVALID_ARG, "hyper is NULL");
    GNN_REQUIRE(hyper->beta1 >= 0.0 && hyper->beta1 < 1.0 && hyper->beta2 >= 0.0 && hyper->beta2 < 1.0, GNN_ERR_INVALID_ARG,
                "beta1 = %g, beta2 = %g: out of [0, 1)", hyper->beta1, hyper->beta2);
    GNN_REQUIRE((float)hyper->eps >= kEpsLeast && (float)hyper->eps <= kEpsMost, GNN_ERR_INVALID_ARG, "eps = %g is out of [%g, %g]", hyper->eps,
                (double)kEpsLeast, (double)kEpsMost);
    // the first step's factor: infinite, it would make a weight that nothing has reached NaN
    GNN_REQUIRE(hyper->lr >= 0.0 && isfinite((float)(hyper->lr / (1.0 - hyper->beta1))), GNN_ERR_INVALID_ARG, "lr = %g: lr / (1 - beta1) is no float", hyper->lr);
    GNN_REQUIRE(state != nullptr || hyper->step >= 1, GNN_ERR_INVALID_ARG, "step = %lld: the first step is 1", (long long)hyper->step);
    GNN_REQUIRE(state != nullptr || isfinite(hyper->grad_scale), GNN_ERR_INVALID_ARG, "grad_scale is not finite");
    GNN_REQUIRE(((uintptr_t)state & 7u) == 0, GNN_ERR_INVALID_ARG, "state is not 8-byte aligned");
    if (n_chunks == 0) return GNN_OK;
    AdamArgs a = {(float)hyper->beta1, (float)(1.0 - hyper->beta1), (float)hyper->beta2, (float)(1.0 - hyper->beta2), (float)hyper->eps,
                  hyper->grad_scale, 0.f, 0.f, hyper->lr, hyper->beta1, hyper->beta2, hyper->step, hyper->rounding_seed};
    if (!state) {
        const double c1 = 1.0 / (1.0 - pow(hyper->beta1, (double)hyper->step));
        a.step_size = (float)(lr_device ? c1 : hyper->lr * c1);    // with lr_device the kernel multiplies
        a.inv_root = (float)(1.0 / sqrt(1.0 - pow(hyper->beta2, (double)hyper->step)));
    }
    if (hyper->rounding_seed) adamw_kernel<true><<<grid_of(n_chunks), 256, 0, (hipStream_t)stream>>>(params, n_params, n_chunks, a, lr_device, state);
    else adamw_kernel<false><<<grid_of(n_chunks), 256, 0, (hipStream_t)stream>>>(params, n_params, n_chunks, a, lr_device, state);
    GNN_LAUNCH_CHECK("adamw_kernel");
    return GNN_OK;
}

extern "C" int32_t gnn_adamw_state_values(const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n, void* m_out,
                                          void* v_out, int32_t dtype, void* stream) {
    GNN_REQUIRE(n >= 0, GNN_ERR_INVALID_ARG, "n < 0");
    GNN_REQUIRE(dtype == GNN_F32 || dtype == GNN_BF16, GNN_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    if (n == 0) return GNN_OK;
    GNN_REQUIRE(m != nullptr && m_scale != nullptr && v != nullptr && v_scale != nullptr && m_out != nullptr && v_out != nullptr,
                GNN_ERR_INVALID_ARG, "NULL argument");
    const bool vec = ((((uintptr_t)m | (uintptr_t)v) & 3u) | (((uintptr_t)m_out | (uintptr_t)v_out) & (dtype == GNN_F32 ? 15u : 7u))) == 0;
    const int grid = grid_for(n, 1024, 8192);
    if (dtype == GNN_F32) state_values_kernel<GNN_F32><<<grid, 256, 0, (hipStream_t)stream>>>(m, m_scale, v, v_scale, n, m_out, v_out, vec);
    else state_values_kernel<GNN_BF16><<<grid, 256, 0, (hipStream_t)stream>>>(m, m_scale, v, v_scale, n, m_out, v_out, vec);
    GNN_LAUNCH_CHECK("state_values_kernel");
    return GNN_OK;
}
