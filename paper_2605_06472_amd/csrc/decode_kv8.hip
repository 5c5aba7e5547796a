// Paged decode attention over an 8-bit pool (one query row per request): every code and scale byte of the context is read exactly once,
// 2 (d + 1) bytes per token and KV head, half of what bf16 rows take.  HBM-bound.
//
// The decomposition is that of the bf16 kernel: a work-group of four waves takes a slice of a request's pages for one KV head and all its
// query heads, a wave every fourth page, its next pages in flight in registers; partial results meet in LDS, those of several slices in the
// last work-group or a second kernel.
//
//   scores     the lane of row c and group g of the 16x16x32 bf16 MFMA's A operand holds eight d of token c.  Which eight is only a label
//              of the contraction, so a lane takes 16 codes with one load (d = 64 j + 16 g ..) and feeds two MFMAs with them, Q^T
//              being loaded in the same order.  Codes become bf16 exactly, two per instruction, without their scale: that
//              multiplies the token's score, of which a lane has four, and not its 8 d.
//   P V        on the 16x16x16 bf16 MFMA, which takes the page's 16 tokens at once: V codes are bf16 numbers, and a probability (times its
//              token's scale) goes in as two, the nearest and what that leaves, 16 bits in all -- an error of 2^-17 of it (at scales near 2^-111 half of
//              bf16's smallest step, 2^-134, where that is more), where the result is rounded to 2^-8.  Against the bf16 kernel's fp32 forms that is as fast up to 4 heads (201 us both for 64 requests of 1024 ..
//              16384 tokens at 32/8 heads of 128), whose 4x4x1 products take as many clocks, and faster past it: 62.4 -> 58.1 at 16/2, 80.4 -> 62.9 at
//              32/2, 36.0 -> 32.3 at 16/2 of 64.  A lane holds d E c .. of four tokens, a word each: four by four bytes are transposed, so that a word is
//              four tokens of one d.  Both scales of its tokens are one 8-byte load.
//   loads      5.8 TB/s of codes at 64 requests of 1024 .. 16384 tokens at 32/8 heads of 128.  What a page's rows take without any arithmetic is
//              197 us of the 201 there; scales, whose line serves four heads on four XCDs, 4 of them.  K rows are read in two halves, which the streaming hint
//              would fetch twice (215 -> 202).
#include "decode_common.h"

#include <algorithm>

namespace pbkv {

#if defined(__HIP_DEVICE_COMPILE__)
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) short i16x4;

template <int D> struct CodeRow;           // the V codes of a lane's D / 16 values of one token
template <> struct CodeRow<128> { typedef u32x2 type; };
template <> struct CodeRow<64> { typedef unsigned type; };

static __device__ __forceinline__ unsigned word(const u32x2 &v, int i) { return v[i]; }
static __device__ __forceinline__ unsigned word(unsigned v, int) { return v; }

// A wave's result to LDS (rows padded by 16 bytes: the lanes of a 16-lane group store 16 bytes to a row each).
template <int D>
static __device__ __forceinline__ void leave_wave(const f32x4 (&acc)[D / 16], float M, float lsum, int G, float *part, float *part_m, float *part_l) {
    constexpr int E = D / 16, PR = D + 4;
    const int g = (threadIdx.x & 63) >> 4, c = threadIdx.x & 15;
    lsum = fold16(lsum, lsum);
    lsum = fold32(lsum, lsum);
    if (c < G) {
        float *ps = part + c * PR + 4 * g * E;
#pragma unroll
        for (int q = 0; q < 4; q++)
#pragma unroll
            for (int e = 0; e < E; e += 4) *(f32x4 *)(ps + q * E + e) = f32x4{acc[e][q], acc[e + 1][q], acc[e + 2][q], acc[e + 3][q]};
    }
    if (c < G && g == 0) {
        part_m[c] = M;
        part_l[c] = lsum;
    }
}

// The four waves of the work-group meet: the result, or the slice's partial, and for FUSED the merge by whoever is last.  part, part_m and
// part_l: what leave_wave left of each wave.
template <int D, bool FUSED>
static __device__ __forceinline__ void finish_slice(const DecodeParams &p, const DecodeReq &rq, int req, int kvh, int slice, int n_slices, int G,
                                                    const float (*part)[DEC_MAX_HEADS * (D + 4)], const float (*part_m)[DEC_MAX_HEADS],
                                                    const float (*part_l)[DEC_MAX_HEADS]) {
    constexpr int PR = D + 4;              // floats of a head's row in LDS
    __syncthreads();
    const int PS = (G * (D + 2) + 3) & ~3;
    const int64_t stride = (int64_t)p.Hkv * PS;                        // between consecutive slices
    float *dst = p.scratch + ((int64_t)(rq.part0 + slice - rq.slice0) * p.Hkv + kvh) * PS;
    __bf16 *out = (__bf16 *)p.out + ((int64_t)req * p.Hq + kvh * G) * D;
    for (int it = threadIdx.x; it < G * D / 4; it += DEC_THREADS) {
        const int h = it * 4 / D, d = it * 4 % D;
        float Mx = -INFINITY, den = 0.f;
#pragma unroll
        for (int ww = 0; ww < DEC_WAVES; ww++) Mx = fmaxf(Mx, part_m[ww][h]);
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ww = 0; ww < DEC_WAVES; ww++) {
            const float f = weight(part_m[ww][h], Mx);
            const f32x4 x = *(const f32x4 *)(part[ww] + h * PR + d);
#pragma unroll
            for (int e = 0; e < 4; e++) num[e] = fmaf(f, x[e], num[e]);
            den = fmaf(f, part_l[ww][h], den);
        }
        if (__builtin_expect(n_slices == 1, 1)) {                      // (laid out first: a partial's stores, the wait behind them and the count are one run)
            bf16x4 r;
#pragma unroll
            for (int e = 0; e < 4; e++) r[e] = (__bf16)normalised(num[e], den);
            *(bf16x4 *)(out + it * 4) = r;
        } else {
            store_partial<FUSED>(dst + it * 4, num[0], num[1]);
            store_partial<FUSED>(dst + it * 4 + 2, num[2], num[3]);
            if (d == 0) store_partial<FUSED>(dst + G * D + 2 * h, Mx, den);
        }
    }
    if constexpr (FUSED) {
        if (n_slices == 1) return;
        // The last work-group to get here merges.  Every thread waits until its stores have been written through to where the other
        // XCDs see them before thread 0 counts the work-group in (which is made there too); the counter wraps to 0 for the next launch on
        // this stream.  The release to the work-group keeps the compiler from moving a store behind the wait; one to the device
        // would write the XCD's whole L2 back.
        __shared__ int is_last;
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0x0F70);                            // vmcnt(0)
        __syncthreads();
        if (threadIdx.x == 0) {
            is_last = atomicInc(p.counters + (int64_t)req * p.Hkv + kvh, (unsigned)n_slices - 1) == (unsigned)n_slices - 1;
        }
        __syncthreads();
        if (!is_last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        // (the host takes this form only where the partials are within MERGE_HELD)
        merge_held<D>(p.scratch + ((int64_t)rq.part0 * p.Hkv + kvh) * PS, stride, n_slices, G, out);
    }
}


// ARGUMENT: the list is `inl`, not in memory.
template <int D, bool FUSED, bool ARGUMENT>
static __device__ __forceinline__ void decode_kv8_slice(const DecodeParams &p, const DecodeList &inl, int G) {
    constexpr int NK = D / 64;             // 16-byte K loads per page, each feeding two MFMAs
    constexpr int E = D / 16;              // d-values of a V row per lane
    constexpr int PR = D + 4;              // floats of a head's row in LDS
    constexpr int BUFS = 2;                // pages of a wave in registers: one being worked on, the next in flight
    typedef typename CodeRow<D>::type vrow;

    const int l = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (all arguments in one trip, and with them the list if it is one of them)
    static_assert(DECODE_INLINE_REQS == 128, "two entries per lane");
    DecodeReq near, far;
    if constexpr (ARGUMENT) near = inl.r[l], far = inl.r[64 + l];
    asm volatile("" ::"s"(p.q), "s"(p.kv_pool), "s"(p.block_table), "s"(p.reqs), "s"(p.mirror_reqs), "s"(p.scratch), "s"(p.n_reqs),
                 "s"(p.slice_pages), "s"(p.Hq), "s"(p.Hkv), "s"(p.max_pages), "s"(p.num_pages), "s"(G));
    const int kvh = blockIdx.x % p.Hkv;
    const int slice = blockIdx.x / p.Hkv;
    int req;
    DecodeReq rq;
    if constexpr (ARGUMENT) {
        req = __builtin_popcountll(__ballot(l < p.n_reqs && near.slice0 <= slice)) +
              __builtin_popcountll(__ballot(64 + l < p.n_reqs && far.slice0 <= slice)) - 1;
        auto pick = [&](int x, int y) {                    // both read: no branch
            const int a = __builtin_amdgcn_readlane(x, req & 63), b = __builtin_amdgcn_readlane(y, req & 63);
            return req < 64 ? a : b;
        };
        rq = DecodeReq{pick(near.ctx_len, far.ctx_len), pick(near.slice0, far.slice0), pick(near.part0, far.part0)};
    } else {
        rq = find_request([&](int i) { return p.reqs[i]; }, p.n_reqs, slice, &req);
    }
    if (p.mirror_reqs != nullptr && kvh == 0 && slice == rq.slice0 && threadIdx.x == 0) p.mirror_reqs[req] = rq;
    const int pages = (rq.ctx_len + 15) >> 4;
    const int n_slices = pages > p.slice_pages ? (pages + p.slice_pages - 1) / p.slice_pages : 1;
    const int page0 = (slice - rq.slice0) * p.slice_pages, page1 = min(pages, page0 + p.slice_pages);
    const int g = l >> 4, c = l & 15;

    // this wave's pages: page0 + w, + 4, ...; their ids sit 64 at a time in one register
    const int32_t *bt = p.block_table + (int64_t)req * p.max_pages;
    const int n_mine = page1 - page0 > w ? (page1 - page0 - w + DEC_WAVES - 1) / DEC_WAVES : 0;
    auto load_ids = [&](int blk) {
        const int k = blk * 64 + l;
        int pg = k < n_mine ? bt[page0 + w + DEC_WAVES * k] : 0;
        return pg < 0 ? 0 : (pg >= p.num_pages ? p.num_pages - 1 : pg);
    };
    int ids = load_ids(0);

    // Q^T operand of MFMA (j, h): lane (g, c) holds q[head c][64 j + 16 g + 8 h .. + 7]; columns >= G are zero
    bf16x8 qB[NK][2];
    {
        const __bf16 *qp = (const __bf16 *)p.q + ((int64_t)req * p.Hq + kvh * G + (c < G ? c : 0)) * D + 16 * g;
#pragma unroll
        for (int j = 0; j < NK; j++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                qB[j][h] = *(const bf16x8 *)(qp + 64 * j + 8 * h);
                if (c >= G) {
#pragma unroll
                    for (int e = 0; e < 8; e++) qB[j][h][e] = (__bf16)0.f;
                }
            }
    }
    const float sc = 1.4426950408889634f * rsqrtf((float)D);   // scores in log2 units

    const int64_t page_bytes = kv8_page_bytes(p.Hkv, D), v_in_page = (int64_t)p.Hkv * 16 * D;
    const char *pool_k = (const char *)p.kv_pool + (int64_t)kvh * 16 * D;
    const char *pool_s = (const char *)p.kv_pool + kv8_codes_bytes(p.Hkv, D) + kvh * 32;
    const int koff = c * D + g * 16;                            // + 64 j
    const int voff = 4 * g * D + c * E;                         // + i * D

    struct PageRegs { u32x4 k[NK]; vrow v[4]; u32x2 s; };
    auto load_page = [&](int k, PageRegs &r) {
        const int64_t at = (int64_t)__builtin_amdgcn_readlane(ids, k & 63) * page_bytes;
        const char *kb = pool_k + at;
        // Every byte is read once, but a line of scales belongs to four KV heads and one of K codes to two of these loads: the streaming hint is on V's alone.
        r.s = *(const u32x2 *)(pool_s + at + 8 * g);
#pragma unroll
        for (int j = 0; j < NK; j++) r.k[j] = *(const u32x4 *)(kb + koff + 64 * j);
#pragma unroll
        for (int i = 0; i < 4; i++) r.v[i] = __builtin_nontemporal_load((const vrow *)(kb + v_in_page + voff + i * D));
    };

    __shared__ __attribute__((aligned(16))) float part[DEC_WAVES][DEC_MAX_HEADS * PR];
    __shared__ float part_m[DEC_WAVES][DEC_MAX_HEADS], part_l[DEC_WAVES][DEC_MAX_HEADS];

    // lane (g, c): acc[e][r] = O[d = E*(4g + r) + e][head c]; reference and partial row sum of head c
    f32x4 acc[E];
#pragma unroll
    for (int e = 0; e < E; e++) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (the lowest finite value, not -inf: keys whose scores are -inf count nothing against it, and the first score that
    // counts is still ahead of it by more than DEC_RESCALE_LOG2)
    float M = -__FLT_MAX__, lsum = 0.f;

    auto compute_page = [&](int k, PageRegs &r) {
        const int valid = rq.ctx_len - (page0 + w + DEC_WAVES * k) * 16;   // >= 1 tokens of this page count
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NK; j++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                bf16x8 a;
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.k[j][2 * h + x], 1.f, false);
                    const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r.k[j][2 * h + x], 1.f, true);
                    a[4 * x] = lo[0]; a[4 * x + 1] = lo[1]; a[4 * x + 2] = hi[0]; a[4 * x + 3] = hi[1];
                }
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qB[j][h], s, 0, 0, 0);
            }
        // lane (g, c): s[i] = score of token 4g + i for head c, without the token's scale.  r.s: K and V scale bytes of tokens 4g .. 4g + 3
        float ks[4], vs[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const unsigned both = r.s[i / 2] >> (16 * (i & 1));
            ks[i] = __uint_as_float((both & 0xff) << 23) * sc;
            vs[i] = __uint_as_float((both >> 8 & 0xff) << 23);
        }
        float t[4];
#pragma unroll
        for (int i = 0; i < 4; i++) t[i] = 4 * g + i < valid ? fmaf(s[i], ks[i], -M) : -INFINITY;
        const float tm = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
        if (__any(c < G && tm > DEC_RESCALE_LOG2)) {
            // move the reference of every head to the largest score the wave has seen
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; i++) mx = fmaxf(mx, 4 * g + i < valid ? s[i] * ks[i] : -INFINITY);
            mx = max_over_head(mx, 16);
            const float newM = fmaxf(M, mx);
            const float alpha = __builtin_amdgcn_exp2f(M - newM);      // 0 on the first page
            M = newM;
            lsum *= alpha;
#pragma unroll
            for (int i = 0; i < 4; i++) t[i] = 4 * g + i < valid ? fmaf(s[i], ks[i], -M) : -INFINITY;
#pragma unroll
            for (int e = 0; e < E; e++) acc[e] *= alpha;
        }
        float pr[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            pr[i] = __builtin_amdgcn_exp2f(t[i]);
            lsum += pr[i];
        }
        if (valid < 16) {
            // slots past the context hold arbitrary codes and scales, which must not reach the product
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (4 * g + i >= valid) {
                    r.v[i] = vrow{};
                    vs[i] = 1.f;
                }
        }
        bf16x4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float x = pr[i] * vs[i];
            hi[i] = (__bf16)x;
            lo[i] = (__bf16)(x - (float)hi[i]);
        }
#pragma unroll
        for (int q = 0; q < E / 4; q++) {
            // four tokens' words of four d each to four words of one d each
            const unsigned a = word(r.v[0], q), b = word(r.v[1], q), c2 = word(r.v[2], q), d2 = word(r.v[3], q);
            const unsigned ab0 = __builtin_amdgcn_perm(b, a, 0x05010400), ab1 = __builtin_amdgcn_perm(b, a, 0x07030602);
            const unsigned cd0 = __builtin_amdgcn_perm(d2, c2, 0x05010400), cd1 = __builtin_amdgcn_perm(d2, c2, 0x07030602);
            const unsigned t[4] = {__builtin_amdgcn_perm(cd0, ab0, 0x05040100), __builtin_amdgcn_perm(cd0, ab0, 0x07060302),
                                   __builtin_amdgcn_perm(cd1, ab1, 0x05040100), __builtin_amdgcn_perm(cd1, ab1, 0x07060302)};
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const bf16x2 v01 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(t[e], 1.f, false), v23 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(t[e], 1.f, true);
                const i16x4 v = __builtin_bit_cast(i16x4, __builtin_shufflevector(v01, v23, 0, 1, 2, 3));
                acc[4 * q + e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, __builtin_bit_cast(i16x4, hi), acc[4 * q + e], 0, 0, 0);
                acc[4 * q + e] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, __builtin_bit_cast(i16x4, lo), acc[4 * q + e], 0, 0, 0);
            }
        }
    };

    // The next page is in flight while one is being worked on.  Behind the last page that one is loaded again (a hit in the caches): where
    // the load hangs on a condition, the waits for a page's rows have to hold without it too, and wait for the next page's.
    PageRegs rg[BUFS];
    if (n_mine > 0) {
#pragma unroll
        for (int b = 0; b < BUFS - 1; b++) load_page(min(b, n_mine - 1), rg[b]);
        for (int k0 = 0;; k0 += BUFS) {
#pragma unroll
            for (int b = 0; b < BUFS; b++) {
                const int k = k0 + b, next = min(k + BUFS - 1, n_mine - 1);
                if (k >= n_mine) goto done;
                if ((next & 63) == 0 && next >= BUFS - 1) ids = load_ids(next >> 6);
                load_page(next, rg[(b + BUFS - 1) % BUFS]);
                compute_page(k, rg[b]);
            }
        }
    }
done:
    leave_wave<D>(acc, M, lsum, G, part[w], part_m[w], part_l[w]);
    finish_slice<D, FUSED>(p, rq, req, kvh, slice, n_slices, G, part, part_m, part_l);
}
#endif

template <int D, bool FUSED, bool ARGUMENT>
__global__ __launch_bounds__(DEC_THREADS) __attribute__((amdgpu_waves_per_eu(D == 128 ? 2 : 4, D == 128 ? 2 : 4)))
void decode_kv8_kernel(DecodeParams p, DecodeList inl, int G) {
#if defined(__HIP_DEVICE_COMPILE__)
    decode_kv8_slice<D, FUSED, ARGUMENT>(p, inl, G);
#endif
}

template <int D>
static hipError_t launch_kv8(const DecodeParams &p, const DecodeList &inl, int G, hipStream_t s) {
    const dim3 grid((unsigned)p.n_slices * p.Hkv);
    const bool list = p.reqs == nullptr, fused = p.counters != nullptr;
    auto kernel = fused ? (list ? decode_kv8_kernel<D, true, true> : decode_kv8_kernel<D, true, false>) : (list ? decode_kv8_kernel<D, false, true> : decode_kv8_kernel<D, false, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(DEC_THREADS), 0, s, p, inl, G);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || fused || p.n_slices == p.n_reqs) return e;          // every request is one slice
    return launch_decode_merge(p, inl, D, s);
}

hipError_t launch_decode_kv8(const DecodeParams &p, const DecodeList &inl, int head_dim, hipStream_t s) {
    const int G = p.Hq / p.Hkv;
    return head_dim == 128 ? launch_kv8<128>(p, inl, G, s) : launch_kv8<64>(p, inl, G, s);
}

}  // namespace pbkv
