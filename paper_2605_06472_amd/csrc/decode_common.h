// What the paged decode kernels share: folds over the lanes of a head, partial results and their merge inside a work-group, and the
// search for a slice's request.
#pragma once
#include "pbkv_internal.h"

namespace pbkv {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;

constexpr int DEC_WAVES = 4;
constexpr int DEC_THREADS = 64 * DEC_WAVES;
[[maybe_unused]] constexpr int DEC_MAX_HEADS = 16;                       // query heads per KV head: the MFMA's columns
[[maybe_unused]] constexpr float DEC_RESCALE_LOG2 = 8.0f;

template <int I> struct IntC { static constexpr int value = I; };

#if defined(__HIP_DEVICE_COMPILE__)
// exp2(m - ref) where m == -inf counts nothing (a wave without pages)
static __device__ __forceinline__ float weight(float m, float ref) { return m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - ref); }

// A row's value.  The sum of its weights is 0 exactly where nothing counts (no tokens, or scores of -inf alone), and the row zero then; a NaN score
// makes it NaN in whatever slice it stands (0 * NaN is NaN, however little the slice weighs), and the row's values with it.
static __device__ __forceinline__ float normalised(float num, float den) { return den == 0.f ? 0.f : num / den; }

// x of this lane and of the lane 32 (16) away, added; lanes whose bit 5 (bit 4) is set get the sum of y instead.
static __device__ __forceinline__ float fold32(float x, float y) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
static __device__ __forceinline__ float fold16(float x, float y) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Over the lanes of a head, which differ in the bits from G up (G a power of two to 16), in every one of them: by exchanges
// inside the vector ALU, where a shuffle goes through LDS (their chain was a sixth of a merge's clocks behind its loads).
template <class Fold>
static __device__ __forceinline__ float over_head(float v, int G, Fold &&fold) {
    auto ror = [&](auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, false)); };
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fold(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fold(__uint_as_float(b[0]), __uint_as_float(b[1]));
    if (G <= 8) v = fold(v, ror(IntC<0x128>{}));           // rotations inside a row of 16 lanes by 8, 4, 2, 1
    if (G <= 4) v = fold(v, ror(IntC<0x124>{}));
    if (G <= 2) v = fold(v, ror(IntC<0x122>{}));
    if (G <= 1) v = fold(v, ror(IntC<0x121>{}));
    return v;
}
static __device__ __forceinline__ float max_over_head(float v, int G) {
    return over_head(v, G, [](float x, float y) { return fmaxf(x, y); });
}
static __device__ __forceinline__ float sum_over_head(float v, int G) {
    return over_head(v, G, [](float x, float y) { return x + y; });
}

// Two neighbouring floats of a partial.  WRITE_THROUGH: past this XCD's L2, for a reader on another one.
template <bool WRITE_THROUGH>
static __device__ __forceinline__ void store_partial(float *dst, float a, float b) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const f32x2 v = {a, b};
    if constexpr (WRITE_THROUGH) {
        uint64_t u;
        __builtin_memcpy(&u, &v, 8);
        __hip_atomic_store((uint64_t *)dst, u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else {
        *(f32x2 *)dst = v;
    }
}

// Merge of the partials of one (request, KV head), normalised and rounded once to bf16, by the threads of a work-group of
// DEC_THREADS.  `base` is slice 0's partial, `stride` the floats between slices.  Which of the two forms below
// serves a (n, G, D) follows from these alone, and so does the order of every sum: the kernel that merges
// does not show in the result.
//
// Up to MERGE_HELD groups of four output values in all (64 KiB of partials, every merge of the one-kernel form): the
// threads load everything at once, 16 groups and one (reference, row sum) each, and weigh what they
// hold: one trip to the other XCDs' stores, which is what a merge of this size costs.  (With references, weights and
// outputs fetched one after the other, 64 output groups at a time, the merge of 16 slices of 4 heads of 128
// took 12000 of a work-group's 22000 clocks: one request of 1003 tokens with append 13.8 -> 11.3 us per pass, 24 of up to
// 4097 at 16/2 heads of 64, where a second kernel merges, 17.7 -> 16.7.)
constexpr int MERGE_HELD = 16 * DEC_THREADS;
template <int D>
static __device__ __forceinline__ void merge_held(const float *base, int64_t stride, int n, int G, __bf16 *out) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    __shared__ float red_m[DEC_WAVES][DEC_MAX_HEADS], red_d[DEC_WAVES][DEC_MAX_HEADS];
    __shared__ float wt[DEC_THREADS];                  // [slice][head]; n * G is at most MERGE_HELD * 4 / D <= 256
    __shared__ __attribute__((aligned(16))) f32x4 red_o[DEC_THREADS];
    const int tid = threadIdx.x;
    const int items = G * D / 4, shift = __builtin_ctz(items), total = n * items;   // a power of two, 16 .. 512
    f32x4 x[MERGE_HELD / DEC_THREADS];
#pragma unroll
    for (int k = 0; k < MERGE_HELD / DEC_THREADS; k++) {
        const int e = k * DEC_THREADS + tid;           // (slice, group)
        x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (e < total) x[k] = *(const f32x4 *)(base + (e >> shift) * stride + (e & (items - 1)) * 4);
    }
    const int h = tid & (G - 1);                       // G divides 64: lanes of one head differ in the bits above G
    f32x2 ml = {-INFINITY, 0.f};
    if (tid / G < n) ml = *(const f32x2 *)(base + (tid / G) * stride + G * D + 2 * h);
    const float m = max_over_head(ml[0], G);
    if ((tid & 63) < G) red_m[tid >> 6][h] = m;
    __syncthreads();
    static_assert(DEC_WAVES == 4, "folds four");
    const float f = weight(ml[0], fmaxf(fmaxf(red_m[0][h], red_m[1][h]), fmaxf(red_m[2][h], red_m[3][h])));
    wt[tid] = f;
    const float d = sum_over_head(f * ml[1], G);
    if ((tid & 63) < G) red_d[tid >> 6][h] = d;
    __syncthreads();
    auto store = [&](int it, const f32x4 &o) {
        const int ho = it * 4 / D;
        const float den = (red_d[0][ho] + red_d[1][ho]) + (red_d[2][ho] + red_d[3][ho]);
        bf16x4 r;
#pragma unroll
        for (int e = 0; e < 4; e++) r[e] = (__bf16)normalised(o[e], den);
        *(bf16x4 *)(out + it * 4) = r;
    };
    f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};      // 512 groups: two per thread; fewer: two chains
#pragma unroll
    for (int k = 0; k < MERGE_HELD / DEC_THREADS; k++) {
        if (k * DEC_THREADS >= total) break;           // uniform
        const int e = k * DEC_THREADS + tid;
        const float we = wt[(e >> shift) * G + (e & (items - 1)) * 4 / D];
#pragma unroll
        for (int c = 0; c < 4; c++) acc[k & 1][c] = fmaf(we, x[k][c], acc[k & 1][c]);
    }
    if (items > DEC_THREADS) {
        store(tid, acc[0]);
        store(tid + DEC_THREADS, acc[1]);
        return;
    }
    f32x4 o = acc[0] + acc[1];
    if (items < DEC_THREADS) {
        red_o[tid] = o;
        __syncthreads();
        if (tid >= items) return;
        for (int k = items + tid; k < DEC_THREADS; k += items) o += red_o[k];
    }
    store(tid, o);
}

// Request that slice `u` belongs to: the last one whose first slice is not behind it.  The whole wave looks at 128
// entries at a time, in two loads that do not wait for each other; longer lists take rounds of 64 before that.
template <class At>
static __device__ __forceinline__ DecodeReq find_request(At &&at, int n, int u, int *req) {
    const int l = threadIdx.x & 63;
    int lo = 0;
    while (n > 128) {
        const int step = (n + 63) / 64;
        const bool before = l * step < n && at(lo + l * step).slice0 <= u;
        const int k = __builtin_popcountll(__ballot(before)) - 1;
        lo += k * step;
        n = min(step, n - k * step);
    }
    const DecodeReq a = at(lo + min(l, n - 1)), b = at(lo + min(64 + l, n - 1));
    const int k = __builtin_popcountll(__ballot(l < n && a.slice0 <= u)) + __builtin_popcountll(__ballot(64 + l < n && b.slice0 <= u)) - 1;
    *req = lo + k;
    const int j = k & 63;
    auto pick = [&](int x, int y) { return k < 64 ? __builtin_amdgcn_readlane(x, j) : __builtin_amdgcn_readlane(y, j); };
    return DecodeReq{pick(a.ctx_len, b.ctx_len), pick(a.slice0, b.slice0), pick(a.part0, b.part0)};
}
#endif

}  // namespace pbkv
