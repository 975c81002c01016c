// Rows of a compressed cache held in 4 bits: the form, and the kernels that gather rows into it and read them back.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace shotkv {

// A unit's rows lie in tiles of 32, the last of which may be partly filled.  An element is x = s (c + z) with a whole code
// c of -8..7, held as the nibble c + 8, and a scale s and a whole z for its group: 32 elements of a key, a value's whole row.
// A tile is its rows' codes in two halves of 16 rows, then a word for each group, s in the high and z in the low 16 bits,
// both bf16.  (Codes and words apart, both parts and so all tiles are multiples of 128 bytes long.)
//
// A half's codes are the A fragments of m16n8k16 products as a warp holds them: word j of lane 4 g + t is that lane's
// fragment of the half's j-th product (words 4 i .. 4 i + 3 of a lane side by side), register p of the fragment nibbles p
// and p + 4.  Keys are 16 rows x 16 dimensions a product, values 16 dimensions x 16 rows.  Which dimension a row or column
// of the product stands for is free, and chosen so that 16 bytes of a bf16 row are 8 elements of one lane:
//   keys     row g + 8 (p & 1),                  dimension 32 (j / 2) + 8 t + 4 (j & 1) + 2 (p >> 1) + e     nibble p + 4 e
//   values   row 2 t + 8 (p >> 1) + e,           dimension 64 (j / 4) + 8 g + 2 (j & 3) + (p & 1)            nibble p + 4 e
template <int D>
struct Kv4 {
    static constexpr int kRows = 32;                       // rows a tile
    static constexpr int kHalfBytes = 16 * D / 2;          // codes of 16 rows
    static constexpr int kCodeBytes = 2 * kHalfBytes;
    static constexpr int kGroups = D / 32;                 // groups of a key
    static constexpr int kKeyTile = kCodeBytes + kRows * kGroups * 4;
    static constexpr int kValueTile = kCodeBytes + kRows * 4;
    static_assert(kKeyTile % 128 == 0 && kValueTile % 128 == 0, "tiles begin on 128-byte boundaries");
};
__host__ __device__ constexpr int kv4_tiles(int rows) { return (rows + 31) / 32; }

// ---- rows into codes ---------------------------------------------------------------------------
// The extremes of some bf16 elements as a pair {max, -min}; NaN if one of them is.
__device__ __forceinline__ uint32_t extremes(uint4 v) {
    const auto b = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    const __nv_bfloat162 mx = __hmax2_nan(__hmax2_nan(b(v.x), b(v.y)), __hmax2_nan(b(v.z), b(v.w)));
    const __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(b(v.x), b(v.y)), __hmin2_nan(b(v.z), b(v.w)));
    const uint32_t hi = *reinterpret_cast<const uint32_t*>(&mx), lo = *reinterpret_cast<const uint32_t*>(&mn) ^ 0x80008000u;
    const __nv_bfloat162 e = __hmax2_nan(b(__byte_perm(hi, lo, 0x5410)), b(__byte_perm(hi, lo, 0x7632)));
    return *reinterpret_cast<const uint32_t*>(&e);
}
__device__ __forceinline__ uint32_t extremes_of(uint32_t a, uint32_t b) {
    const __nv_bfloat162 e = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&e);
}

// What a group's elements are turned into codes with: the fused product x * inv + shift is a number of [2048, 4096) whose
// whole part ends in the code + 8's four bits.
struct Grid4 {
    float inv, shift;
    uint32_t word;       // s and z as they are kept
};
// The scale is the least bf16 number s with 15 s >= R = max(range, max|x| / 16, 15 * 2^-100): sixteen steps reach
// over the range, the grid of multiples of s is no finer than bf16 itself near the group's largest element (so that z is
// whole and below 256, exact in bf16), and nothing is divided by zero.  c + z = floor(x / s + 1/2).
// The range is that of the numbers themselves, which 32 bits may round.  15 s has 12 bits, so it is on the same side of the range as of the
// rounded one, unless it is the rounded one: then what was rounded off decides.  (It is exact in 32 bits: of max and -min the greater is
// no smaller in magnitude than the other.)
// A quotient x / s of bf16 numbers that the rule admits (|x / s| <= 240) is a half-integer or 2^-10 away from every one, so
// a quotient off by less (1 / s to 2^-22, the sum rounded to 2^-12) is rounded the right way once 2^-12 is added.
__device__ __forceinline__ Grid4 grid_of(uint32_t extreme) {
    const float mx = __uint_as_float(extreme << 16), neg = __uint_as_float(extreme & 0xffff0000u);    // max and -min
    const float sum = mx + neg, most = fmaxf(mx, neg), rest = fminf(mx, neg) - (sum - most);
    const float R = fmaxf(fmaxf(sum, most * 0.0625f), 15.f * 0x1p-100f);
    // 1/15 rounded down, and the product down to bf16; then up until it is enough (products with 15 are exact)
    uint32_t s = __float_as_uint(R * 0x1.11111p-4f) & 0xffff0000u;
    if (__uint_as_float(s) * 15.f < R) s += 0x10000u;
    if (__uint_as_float(s) * 15.f < R) s += 0x10000u;
    if (__uint_as_float(s) * 15.f == sum && rest > 0.f) s += 0x10000u;
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(__uint_as_float(s)));
    const float base = 2560.5f + 0x1p-12f;
    // an element that is not finite, or a range beyond float32 (fmaxf drops a NaN, the sum keeps it): the whole group reads as NaN
    const bool fine = sum < __int_as_float(0x7f800000);
    if (!fine) inv = 0.f;
    const float z = __uint_as_float(__float_as_uint(fine ? fmaf(-neg, inv, base) : base) & 0xfffff000u) - 2560.f;
    Grid4 g;
    g.inv = inv;
    g.shift = base - z;
    g.word = (fine ? s : 0x7fc00000u) | (__float_as_uint(z + 8.f) >> 16);
    return g;
}
__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Eight numbers as grid_of's products leave them, register p's pair (lo[p], hi[p]), as a word of codes.
__device__ __forceinline__ uint32_t codes_word(const float (&lo)[4], const float (&hi)[4]) {
    uint32_t P[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) P[p] = __byte_perm(__float_as_uint(lo[p]), __float_as_uint(hi[p]), 0x5410);
    return ((P[0] >> 12) & 0x000f000fu) | ((P[1] >> 8) & 0x00f000f0u) | ((P[2] >> 4) & 0x0f000f00u) | (P[3] & 0xf000f000u);
}

// Row gather into the packed form: row j of a unit is row kept_idx[bl][j] of K and V (row j itself without indices).  Rows
// from the count on in the last tile become rows of zeros; later tiles are left as they are.  A warp takes 16 rows:
// sixteen 16-byte loads a lane in flight, and what it loads are the very elements of its own code words, so that nothing
// goes through shared memory.  The lanes that hold a group's elements fold their extremes together and each works out
// the grid of other groups.  grid = (warps' halves of a unit, Hkv, B*L).
// HBM-bound: 32 layers of 16,384 tokens, a fifth of them kept, 83 us, 6.25 TB/s read and written (in CTAs of 256 threads, of
// which two fit an SM, 93).
constexpr int kPackThreads = 128;
template <int D>
__global__ void __launch_bounds__(kPackThreads) compact_kv4_kernel(const uint4* K, const uint4* V, const int* kept_idx, const int* kept_count,
                                                                  int Hkv, int N, int Mcap, unsigned char* K4, unsigned char* V4) {
    using F = Kv4<D>;
    constexpr int VPR = D / 8, NB = D / 32, NC = D / 64;   // 16-byte vectors a row, 32- and 64-dimension blocks
    const int bl = blockIdx.z, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int half = blockIdx.x * (kPackThreads / 32) + (threadIdx.x >> 5), row0 = half * 16;
    grid_release();
    grid_wait();
    const int j = row0 + (lane & 15);
    int src = kept_idx && j < Mcap ? kept_idx[(size_t)bl * Mcap + j] : j;
    const int count = min(kept_count[bl], Mcap);
    if (row0 >= count && ((half & 1) == 0 || row0 - 16 >= count)) return;    // nothing in this tile
    if (j >= count || src >= N) src = -1;
    const size_t u = (size_t)bl * Hkv + blockIdx.y;
    const uint4 *Ku = K + u * N * VPR, *Vu = V + u * N * VPR;

    const int s0 = __shfl_sync(0xffffffffu, src, g), s1 = __shfl_sync(0xffffffffu, src, g + 8);
    uint4 k[2 * NB], v[4 * NC];                            // k[i * NB + kb]: row g + 8 i;  v[c * 4 + i]: the i-th of the lane's four rows
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
        k[kb] = load_if(Ku + (ptrdiff_t)s0 * VPR + kb * 4 + t, s0 >= 0);
        k[NB + kb] = load_if(Ku + (ptrdiff_t)s1 * VPR + kb * 4 + t, s1 >= 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int sv = __shfl_sync(0xffffffffu, src, 2 * t + (i & 1) + 8 * (i >> 1));
#pragma unroll
        for (int c = 0; c < NC; ++c) v[c * 4 + i] = load_if(Vu + (ptrdiff_t)sv * VPR + c * 8 + g, sv >= 0);
    }

    unsigned char* Kt = K4 + (u * kv4_tiles(Mcap) + (half >> 1)) * F::kKeyTile;
    unsigned char* Vt = V4 + (u * kv4_tiles(Mcap) + (half >> 1)) * F::kValueTile;
    {   // keys: group (row g + 8 i, kb) lies in the four lanes of a g, and its grid is worked out by lane (i * NB + kb) % 4
        uint32_t e[2 * NB];
#pragma unroll
        for (int x = 0; x < 2 * NB; ++x) {
            e[x] = extremes(k[x]);
            e[x] = extremes_of(e[x], __shfl_xor_sync(0xffffffffu, e[x], 1));
            e[x] = extremes_of(e[x], __shfl_xor_sync(0xffffffffu, e[x], 2));
        }
        Grid4 mine[NB / 2];
#pragma unroll
        for (int y = 0; y < NB / 2; ++y) {
            const uint32_t a = t & 1 ? e[4 * y + 1] : e[4 * y], b = t & 1 ? e[4 * y + 3] : e[4 * y + 2];
            mine[y] = grid_of(t & 2 ? b : a);
            const int i = NB == 4 ? y : t >> 1, kb = NB == 4 ? t : t & 1;
            reinterpret_cast<uint32_t*>(Kt + F::kCodeBytes)[((half & 1) * 16 + g + 8 * i) * NB + kb] = mine[y].word;
        }
        uint32_t w[2 * NB];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            float inv[2], shift[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int x = i * NB + kb;
                inv[i] = __shfl_sync(0xffffffffu, mine[x / 4].inv, (lane & ~3) + x % 4);
                shift[i] = __shfl_sync(0xffffffffu, mine[x / 4].shift, (lane & ~3) + x % 4);
            }
            const auto word = [&](uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
                const float lo[4] = {fmaf(bf16_low(a0), inv[0], shift[0]), fmaf(bf16_low(b0), inv[1], shift[1]),
                                     fmaf(bf16_low(a1), inv[0], shift[0]), fmaf(bf16_low(b1), inv[1], shift[1])};
                const float hi[4] = {fmaf(bf16_high(a0), inv[0], shift[0]), fmaf(bf16_high(b0), inv[1], shift[1]),
                                     fmaf(bf16_high(a1), inv[0], shift[0]), fmaf(bf16_high(b1), inv[1], shift[1])};
                return codes_word(lo, hi);
            };
            const uint4 a = k[kb], b = k[NB + kb];
            w[2 * kb] = word(a.x, a.y, b.x, b.y);
            w[2 * kb + 1] = word(a.z, a.w, b.z, b.w);
        }
        uint4* to = reinterpret_cast<uint4*>(Kt + (half & 1) * F::kHalfBytes);
#pragma unroll
        for (int c = 0; c < NC; ++c) to[c * 32 + lane] = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
    }
    {   // values: row 2 t + (i & 1) + 8 (i >> 1) lies in the eight lanes of a t, and lanes g and g + 4 work out row i = g % 4's grid
        uint32_t e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = extremes(v[i]);
            if (NC == 2) e[i] = extremes_of(e[i], extremes(v[4 * (NC - 1) + i]));
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) e[i] = extremes_of(e[i], __shfl_xor_sync(0xffffffffu, e[i], o));
        }
        const uint32_t a = g & 1 ? e[1] : e[0], b = g & 1 ? e[3] : e[2];
        const Grid4 mine = grid_of(g & 2 ? b : a);
        if (g < 4) reinterpret_cast<uint32_t*>(Vt + F::kCodeBytes)[(half & 1) * 16 + 2 * t + (g & 1) + 8 * (g >> 1)] = mine.word;
        float inv[4], shift[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            inv[i] = __shfl_sync(0xffffffffu, mine.inv, 4 * i + t);
            shift[i] = __shfl_sync(0xffffffffu, mine.shift, 4 * i + t);
        }
        const auto word = [&](uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
            const float lo[4] = {fmaf(bf16_low(r0), inv[0], shift[0]), fmaf(bf16_high(r0), inv[0], shift[0]),
                                 fmaf(bf16_low(r2), inv[2], shift[2]), fmaf(bf16_high(r2), inv[2], shift[2])};
            const float hi[4] = {fmaf(bf16_low(r1), inv[1], shift[1]), fmaf(bf16_high(r1), inv[1], shift[1]),
                                 fmaf(bf16_low(r3), inv[3], shift[3]), fmaf(bf16_high(r3), inv[3], shift[3])};
            return codes_word(lo, hi);
        };
        uint4* to = reinterpret_cast<uint4*>(Vt + (half & 1) * F::kHalfBytes);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 r0 = v[4 * c], r1 = v[4 * c + 1], r2 = v[4 * c + 2], r3 = v[4 * c + 3];
            to[c * 32 + lane] = make_uint4(word(r0.x, r1.x, r2.x, r3.x), word(r0.y, r1.y, r2.y, r3.y), word(r0.z, r1.z, r2.z, r3.z),
                                           word(r0.w, r1.w, r2.w, r3.w));
        }
    }
}

// ---- codes into numbers ------------------------------------------------------------------------
// (w & MASK) | under as the one instruction it is (written out, its two constants made two of it).
template <uint32_t MASK>
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t under) {
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(w), "n"(MASK), "r"(under));
    return d;
}
// What codes are put under: 1024 and 1032, as pairs of f16.
struct Under {
    uint32_t k1024, k1032;
};
__device__ __forceinline__ Under codes_under() { return Under{0x64006400u, 0x64086408u}; }
// A word's four registers of an A fragment: pairs of codes -8..7 as f16, of registers 1 and 3 sixteen times as much, exact.
// A byte under the significand of 1024 is 1024 + n + 16 n', its upper nibble under that of 1032 is 1032 + 16 n': their
// difference is n - 8, and the second less 1160 is 16 (n' - 8).  (Eight instructions a word, four of them on the pipe of the logical
// operations; each nibble by itself under 1024 takes nine and five.)
__device__ __forceinline__ void codes_f16(uint32_t w, const Under& k, uint32_t (&a)[4]) {
    const auto h = [](uint32_t x) { return *reinterpret_cast<const __half2*>(&x); };
    const auto u = [](__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); };
    const __half2 less = h(0xe488e488u);                                  // -1160
    const uint32_t low = and_or<0x00ff00ffu>(w, k.k1024), high = __byte_perm(w, k.k1024, 0x5351);
    const uint32_t low1 = and_or<0x00f000f0u>(w, k.k1032), high1 = and_or<0x00f000f0u>(high, k.k1032);
    a[0] = u(__hsub2(h(low), h(low1)));
    a[1] = u(__hadd2(h(low1), less));
    a[2] = u(__hsub2(h(high), h(high1)));
    a[3] = u(__hadd2(h(high1), less));
}
// The same as f16 subnormals: code + 8 in units of 2^-24, of registers 1 and 3 (rows g + 8 of a product) of 2^-20.
__device__ __forceinline__ void codes_subnormal(uint32_t w, uint32_t (&a)[4]) {
    const uint32_t v = w >> 8;
    a[0] = w & 0x000f000fu, a[1] = w & 0x00f000f0u, a[2] = v & 0x000f000fu, a[3] = v & 0x00f000f0u;
}

// The packed rows below the count as bf16, each element rounded once: a warp takes 16 rows, as above (81 us for the same rows,
// 6.4 TB/s).
template <int D>
__global__ void __launch_bounds__(kPackThreads) unpack_kv4_kernel(const unsigned char* K4, const unsigned char* V4, const int* kept_count, int Hkv,
                                                                 int Mcap, uint4* Kc, uint4* Vc) {
    using F = Kv4<D>;
    constexpr int VPR = D / 8, NB = D / 32, NC = D / 64;
    const int bl = blockIdx.z, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int half = blockIdx.x * (kPackThreads / 32) + (threadIdx.x >> 5), row0 = half * 16;
    grid_release();
    grid_wait();
    const int count = min(kept_count[bl], Mcap);
    if (row0 >= count) return;
    const size_t u = (size_t)bl * Hkv + blockIdx.y;
    const unsigned char* Kt = K4 + (u * kv4_tiles(Mcap) + (half >> 1)) * F::kKeyTile;
    const unsigned char* Vt = V4 + (u * kv4_tiles(Mcap) + (half >> 1)) * F::kValueTile;
    const uint32_t *Km = reinterpret_cast<const uint32_t*>(Kt + F::kCodeBytes) + (half & 1) * 16 * NB,
                   *Vm = reinterpret_cast<const uint32_t*>(Vt + F::kCodeBytes) + (half & 1) * 16;
    uint4 kw[NC], vw[NC];
    uint32_t km[2 * NB], vm[4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        kw[c] = reinterpret_cast<const uint4*>(Kt + (half & 1) * F::kHalfBytes)[c * 32 + lane];
        vw[c] = reinterpret_cast<const uint4*>(Vt + (half & 1) * F::kHalfBytes)[c * 32 + lane];
    }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) km[kb] = Km[g * NB + kb], km[NB + kb] = Km[(g + 8) * NB + kb];
#pragma unroll
    for (int i = 0; i < 4; ++i) vm[i] = Vm[2 * t + (i & 1) + 8 * (i >> 1)];
    const auto value = [](float c, uint32_t m) { return bf16_high(m) * (c + bf16_low(m)); };
    const Under under = codes_under();
    const auto pair = [](float a, float b) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    };
    const auto split = [](uint32_t a) { return __half22float2(*reinterpret_cast<const __half2*>(&a)); };
    uint4* Kr = Kc + (u * Mcap + row0) * VPR;
    uint4* Vr = Vc + (u * Mcap + row0) * VPR;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {                      // the lane's 16 bytes of rows g and g + 8
        uint32_t r[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 w4 = kw[kb / 2];
            uint32_t a[4];
            codes_f16(kb & 1 ? (h ? w4.w : w4.z) : (h ? w4.y : w4.x), under, a);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                float2 c = split(a[p]);
                if (p & 1) c.x *= 0.0625f, c.y *= 0.0625f;
                const uint32_t m = km[(p & 1) * NB + kb];
                r[p & 1][2 * h + (p >> 1)] = pair(value(c.x, m), value(c.y, m));
            }
        }
        if (row0 + g < count) Kr[g * VPR + kb * 4 + t] = make_uint4(r[0][0], r[0][1], r[0][2], r[0][3]);
        if (row0 + g + 8 < count) Kr[(g + 8) * VPR + kb * 4 + t] = make_uint4(r[1][0], r[1][1], r[1][2], r[1][3]);
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {                         // the lane's 16 bytes of its four rows
        uint32_t r[4][4];
        const uint32_t w4[4] = {vw[c].x, vw[c].y, vw[c].z, vw[c].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[4];
            codes_f16(w4[i], under, a);
#pragma unroll
            for (int h = 0; h < 2; ++h) {                  // rows 2 t + 8 h and the next
                const float2 even = split(a[2 * h]), odd = split(a[2 * h + 1]);
                r[2 * h][i] = pair(value(even.x, vm[2 * h]), value(odd.x * 0.0625f, vm[2 * h]));
                r[2 * h + 1][i] = pair(value(even.y, vm[2 * h + 1]), value(odd.y * 0.0625f, vm[2 * h + 1]));
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 2 * t + (i & 1) + 8 * (i >> 1);
            if (row0 + row < count) Vr[row * VPR + c * 8 + g] = make_uint4(r[i][0], r[i][1], r[i][2], r[i][3]);
        }
    }
}

}  // namespace shotkv
