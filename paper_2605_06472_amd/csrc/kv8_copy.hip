// K/V rows on their way into an 8-bit pool and back: bf16 rows are quantised to e4m3 codes with one power-of-two scale each, and
// come back as the bf16 numbers that the codes stand for.
//
//   scale   2^e, the smallest power of two with which the row's largest finite magnitude is at most 448, e4m3's largest number:
//           with a = 1.m 2^E, e = E - 8 where 1.m <= 1.75 and E - 7 elsewhere, within [KV8_MIN_EXP, KV8_MAX_EXP].
//   code    x 2^-e rounded to the nearest e4m3 number, ties to even.  Above 448 2^KV8_MAX_EXP (within a factor of 1.14 of bf16's
//           largest number) it saturates.  Infinities and NaN become NaN, so that attention over the row shows them as a bf16 pool would.
// A power of two costs nothing against a finer scale: e4m3 is a floating-point format, whose relative step (2^-3 of a value's own power of
// two) does not depend on where in its range a row lies, and it is what makes the way back exact.
//
// Both are copies, bound by memory: 4 d bytes of bf16 per token and head on one side, 2 d + 2 on the other.  An item is 16 values of a row of
// K and the same of V, eight of each half of the row: so that the lanes of a row store and load 16-byte words of bf16, and 8-byte words of codes, side by side.
// With 16 values in a run a store instruction writes every other 16 bytes, and streaming stores then reach memory in parts (1.28 times the
// bytes that are there to write): 32768 tokens of 8 heads of 128, append 37.4 -> 32.5 us, read 39.7 -> 31.7 (6.4 TB/s; 4.9 is what a copy
// of 2 GiB reaches); read of 12001 15.9 -> 10.6.  Both scales are one 16-bit word.  The D / 16 lanes of a row find its largest magnitude by exchanges in the
// vector ALU.
// Streaming hints where they were measured to pay: stores (append of 8 requests of 500 .. 1500 tokens 6.5 -> 5.5 us, of 32768 the same; read of 12001 12.9 ->
// 10.6) and no load: a line of codes is read by two instructions (read 10.6, with the hint 15.4), and the rows to be appended are
// best read as if their producer had just left them in a cache (append of 32768 35.5 with the hint, 32.5).
#include "pbkv_internal.h"

namespace pbkv {

typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) short i16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// Work-groups of a launch: one per part, where the copy kernels of plain rows hold a grid of the chip's size that strides over them.  A work-group has one trip's
// loads and is gone; the dispatcher evens out what a second, half empty round leaves idle.  us, 2048 and one per part: append of 32768 tokens of 8 heads of
// 128 33.0, 32.6, read 32.1, 31.7; of 2 requests of 3000 .. 5000 of 32 heads 32.0, 30.8 and 30.2, 29.6.
constexpr int KV8_MAX_WGS = 1 << 20;

#if defined(__HIP_DEVICE_COMPILE__)
static __device__ __forceinline__ int clamp_page(int pg, int num_pages) {
    return pg < 0 ? 0 : (pg >= num_pages ? num_pages - 1 : pg);
}

struct Row16 { u32x4 a, b; };       // 16 bf16 values

// Largest of the 16-bit magnitudes over the D / 16 lanes of a row, in all of them.
template <int D>
static __device__ __forceinline__ unsigned over_row(unsigned v) {
    auto max_u = [](unsigned a, unsigned b) { return a > b ? a : b; };
    v = max_u(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));                            // the neighbour
    v = max_u(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));                            // the other pair of four
    if constexpr (D == 128) v = max_u(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));   // the other four of eight
    return v;
}

static __device__ __forceinline__ unsigned magnitudes(const Row16 &x) {
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned a = x.a[i] & 0x7fff7fffu, b = x.b[i] & 0x7fff7fffu;
        m = __builtin_elementwise_max(m, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    return m[0] > m[1] ? m[0] : m[1];
}

constexpr unsigned BF16_INF = 0x7f80, KV8_TOP = 0x7f60;     // infinity; 448 2^KV8_MAX_EXP

// Codes of this lane's 16 values, and the row's scale byte.
template <int D>
static __device__ __forceinline__ u32x4 quantise(const Row16 &x, unsigned *scale_byte) {
    unsigned top = over_row<D>(magnitudes(x));
    const bool plain = top <= KV8_TOP;
    if (!plain) {
        // infinities, NaN, or finite values that the scales do not reach: the largest finite magnitude
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const unsigned w = (i < 4 ? x.a[i & 3] : x.b[i & 3]) & 0x7fff7fffu, lo = w & 0xffff, hi = w >> 16;
            if (lo < BF16_INF) m = m > lo ? m : lo;
            if (hi < BF16_INF) m = m > hi ? m : hi;
        }
        top = over_row<D>(m);
    }
    // (a zero or subnormal row's exponent field is 0: far below the smallest scale)
    int e = (int)(top >> 7) - 127 - 8 + ((top & 0x7f) > 0x60);
    e = e < KV8_MIN_EXP ? KV8_MIN_EXP : (e > KV8_MAX_EXP ? KV8_MAX_EXP : e);
    *scale_byte = (unsigned)(e + 127);
    const float scale = __uint_as_float((unsigned)(e + 127) << 23);
    u32x4 codes;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        auto word = [&](int k) { return k < 4 ? x.a[k] : x.b[k - 4]; };
        unsigned lo = word(2 * i), hi = word(2 * i + 1);
        if (!plain) {
            // finite values past the largest code's become it (the conversion would give NaN); a NaN goes in as the infinity of its sign
            auto limit = [](unsigned a) { return a > BF16_INF ? BF16_INF : a < BF16_INF && a > KV8_TOP ? KV8_TOP : a; };
            auto saturate = [&](unsigned w) { return (w & 0x80008000u) | limit(w & 0x7fff) | limit((w >> 16) & 0x7fff) << 16; };
            lo = saturate(lo);
            hi = saturate(hi);
        }
        i16x2 c = {0, 0};
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, lo), scale, false);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, __builtin_bit_cast(bf16x2, hi), scale, true);
        codes[i] = __builtin_bit_cast(unsigned, c);
    }
    return codes;
}

static __device__ __forceinline__ Row16 values(const u32x4 &codes, float scale) {
    Row16 x;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned lo = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, false));
        const unsigned hi = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[i], scale, true));
        if (i < 2) x.a[2 * i] = lo, x.a[2 * i + 1] = hi;
        else x.b[2 * i - 4] = lo, x.b[2 * i - 3] = hi;
    }
    return x;
}
#endif

// Work: runs of up to 16 tokens of one request in one page, cut into parts of 256 items; an item's number counts lanes of a row, heads, tokens,
// in the packed rows' order.
template <int D, bool READ>
__global__ __launch_bounds__(256) void kv8_copy_kernel(AppendParams p, unsigned parts_per_run, int step_runs, unsigned step_parts) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int LPR = D / 16;                               // lanes of a row
    const int64_t page_bytes = kv8_page_bytes(p.Hkv, D), codes_bytes = kv8_codes_bytes(p.Hkv, D);
    int run = (int)(blockIdx.x / parts_per_run);
    unsigned part_u = blockIdx.x % parts_per_run;
    for (; run < p.n_descs; run += step_runs, part_u += step_parts, run += part_u >= parts_per_run, part_u -= part_u >= parts_per_run ? parts_per_run : 0) {
        const int part = (int)part_u;
        const AppendDesc d = p.descs[run];
        if (p.mirror != nullptr && part == 0 && threadIdx.x == 0) p.mirror[run] = d;
        const int total = d.count * p.Hkv * LPR;
        const int idx = part * 256 + (int)threadIdx.x;
        if (idx >= total) continue;                           // (whole rows: the lanes of a row stay together)
        const int page_id = p.block_table[(int64_t)d.req * p.max_pages + d.logical_page];
        const int c = idx % LPR;
        const unsigned row = (unsigned)idx / LPR, t = row / (unsigned)p.Hkv;
        const int g = (int)(row - t * p.Hkv), slot = d.slot0 + (int)t;
        const int64_t packed = ((d.src_row + t) * p.Hkv + g) * (D / 8) + c;           // 16-byte words
        char *page = (char *)p.kv_pool + (int64_t)clamp_page(page_id, p.num_pages) * page_bytes;
        u32x2 *kc = (u32x2 *)(page + ((int64_t)g * 16 + slot) * D) + c;
        u32x2 *vc = (u32x2 *)(page + ((int64_t)(p.Hkv + g) * 16 + slot) * D) + c;
        uint16_t *sc = (uint16_t *)(page + codes_bytes) + g * 16 + slot;
        u32x4 *kp = (u32x4 *)p.k_new + packed, *vp = (u32x4 *)p.v_new + packed;
        if constexpr (READ) {
            const u32x2 k0 = kc[0], k1 = kc[LPR], v0 = vc[0], v1 = vc[LPR];
            const unsigned s = *sc;
            const Row16 x = values(u32x4{k0[0], k0[1], k1[0], k1[1]}, __uint_as_float((s & 0xff) << 23));
            const Row16 y = values(u32x4{v0[0], v0[1], v1[0], v1[1]}, __uint_as_float((s >> 8) << 23));
            __builtin_nontemporal_store(x.a, kp);
            __builtin_nontemporal_store(x.b, kp + LPR);
            __builtin_nontemporal_store(y.a, vp);
            __builtin_nontemporal_store(y.b, vp + LPR);
        } else {
            const Row16 x = {kp[0], kp[LPR]}, y = {vp[0], vp[LPR]};
            unsigned ks, vs;
            const u32x4 k = quantise<D>(x, &ks), v = quantise<D>(y, &vs);
            __builtin_nontemporal_store(u32x2{k[0], k[1]}, kc);
            __builtin_nontemporal_store(u32x2{k[2], k[3]}, kc + LPR);
            __builtin_nontemporal_store(u32x2{v[0], v[1]}, vc);
            __builtin_nontemporal_store(u32x2{v[2], v[3]}, vc + LPR);
            if (c == 0) *sc = (uint16_t)(ks | vs << 8);
        }
    }
#endif
}

template <bool READ>
static hipError_t launch_copy(const AppendParams &p, int head_dim, hipStream_t s) {
    if (p.n_descs == 0) return hipSuccess;
    const int parts = (16 * p.Hkv * (head_dim / 16) + 255) / 256;
    const int64_t items = (int64_t)p.n_descs * parts;
    const int grid = (int)(items < KV8_MAX_WGS ? items : KV8_MAX_WGS);
    if (head_dim == 128) hipLaunchKernelGGL((kv8_copy_kernel<128, READ>), dim3((unsigned)grid), dim3(256), 0, s, p, (unsigned)parts, grid / parts, (unsigned)(grid % parts));
    else hipLaunchKernelGGL((kv8_copy_kernel<64, READ>), dim3((unsigned)grid), dim3(256), 0, s, p, (unsigned)parts, grid / parts, (unsigned)(grid % parts));
    return hipGetLastError();
}

hipError_t launch_append_kv8(const AppendParams &p, int head_dim, hipStream_t s) { return launch_copy<false>(p, head_dim, s); }
hipError_t launch_read_kv8(const AppendParams &p, int head_dim, hipStream_t s) { return launch_copy<true>(p, head_dim, s); }

}  // namespace pbkv
