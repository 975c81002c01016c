// The decode steps over a prompt's cache held in 4 bits (kv4.cuh).
#pragma once
#include <type_traits>

#include "decode.cuh"
#include "kv4.cuh"

namespace shotkv {

// D(16x8,f32) += A(16x16,f16,row) * B(16x8,f16,col)
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8x8 matrix of 16-bit elements, two neighbours of row lane / 4 a lane, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t a) { return __half22float2(*reinterpret_cast<const __half2*>(&a)); }

struct PackedCache {
    const unsigned char *K4, *V4;            // [U][tiles][Kv4 tile]
};

template <int D, bool ATTEND>
struct StepKv4 {
    static constexpr int kWarps = 4;
    static constexpr int kStages = ATTEND ? 2 : 3;         // tiles in a warp's ring
    static constexpr int kStageBytes = Kv4<D>::kKeyTile + (ATTEND ? Kv4<D>::kValueTile : 0);
    static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
    static_assert(!ATTEND || 8 * kOutPitch<D> * 4 <= kStages * kStageBytes, "a warp's outputs take the place of its ring");
};
template <int D, bool ATTEND>
__host__ __device__ constexpr size_t kv4_smem_bytes(int G, int Dcap, int nsplit) {
    const size_t shares = nsplit > 1 ? (size_t)nsplit * (16 + (ATTEND ? (G * D / 4 / nsplit + 1) * 4 : 0)) : 0;
    return StepKv4<D, ATTEND>::kRingBytes + 16 + ((size_t)StepKv4<D, ATTEND>::kWarps * 16 + ((size_t)G * Dcap + 3) / 4 * 4 + shares) * 4;
}

// decode_score_kernel's and (ATTEND) decode_attend_kernel's step over packed prefill rows.  A warp takes decode entries,
// which are bf16, 16 at a time straight from global memory, and packed rows a tile of 32 at a time through its ring.
//
// Both products have the keys, or the values' dimensions, on the 16-row side, so that a packed word is an operand's
// fragment but for the conversion, and the group's (up to 8) query rows on the side of 8:
//   S[16 keys x 8 rows] = codes . q, one chain of products for every group of 32 dimensions, in f16: codes are whole numbers, and
//     a query row, bf16, is multiplied by the power of two that takes its largest element to [2^14, 2^15), which leaves elements
//     down to 2^-31 of it exact.  A logit is sum over groups s (S + z sum of q's 32 elements).
//   O^T[16 dims x 8 rows] += codes^T . w^T with w = p s_v, p = 2^(logit - reference): the accumulator of S, transposed 8 by 8, is
//     the other operand, an f16 pair (high part and remainder: 2^-22 of w, or 2^-35 of the row's largest where that is more).  z
//     is added once a row: sum of w z_v.
//
// f16 ends at 65504, so both factors are kept in range by references that change seldom: a row's reference is 2^10 below its
// maximum when it was last set and is set again by a tile whose p would exceed 2^13, and the values' scales are multiplied by a
// power of two that takes the largest of the first tile to [1, 2) and is set again when one exceeds 4.  One vote a
// half tile decides that neither has happened.
template <int D, bool ATTEND, bool FUSED>
__global__ void __launch_bounds__(StepKv4<D, ATTEND>::kWarps * 32, 4)
decode_kv4_kernel(const DecodeParams p, const DecodeFinishParams f, const PackedCache cache) {
    using Cfg = StepKv4<D, ATTEND>;
    using F = Kv4<D>;
    constexpr int NB = D / 32, NC = D / 64, VPR = D / 8, MT = D / 16;
    constexpr int NW = Cfg::kWarps, NS = Cfg::kStages;
    constexpr float kLift = 10.f, kHighest = 13.f, kUnset = -1e30f;
    extern __shared__ __align__(128) unsigned char dsm[];
    unsigned char* ring = dsm;                               // [NW][NS][keys | values]; later each warp's outputs
    float2* sred = reinterpret_cast<float2*>(ring + Cfg::kRingBytes + 16);   // [NW warps][8 rows]  (m, z)
    float* sdec = reinterpret_cast<float*>(sred + NW * 8);   // [G][Dcap]  logits of the decode entries
    float2* stab = reinterpret_cast<float2*>(sdec + ((p.G * p.Dcap + 3) & ~3));
    float4* sin = reinterpret_cast<float4*>(stab + p.nsplit * 8);
    unsigned long long* arrived = reinterpret_cast<unsigned long long*>(sred) - 1;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t4 = lane & 3;
    const int u = blockIdx.x / p.nsplit, rank = blockIdx.x - u * p.nsplit;
    const QuadShare qs = quads_of<D>(p.G, p.nsplit, rank);
    const int bl = u / p.Hkv, hk = u - bl * p.Hkv;
    const int first_cta = FUSED ? hk * p.nsplit : 0, ctas = p.Hkv * p.nsplit;   // in the cluster: the unit's first; FUSED: all
    FusedEnd end{};
    if (FUSED) end = fused_end_at(dsm + kv4_smem_bytes<D, ATTEND>(p.G, p.Dcap, p.nsplit), f);
    if (FUSED || p.nsplit > 1) {
        if (tid == 0) {
            if (p.nsplit > 1) expect_messages(arrived, p.nsplit * (8 * (int)sizeof(float2) + (ATTEND ? qs.owned * (int)sizeof(float4) : 0)));
            if (FUSED) fused_expect(end, f, first_cta + rank);
        }
        cluster_arrive();
    }
    grid_wait();
    grid_release();
    uint4* Kd_u = reinterpret_cast<uint4*>(p.Kd + (size_t)u * p.Dcap * D);
    uint4* Vd_u = reinterpret_cast<uint4*>(p.Vd + (size_t)u * p.Dcap * D);
    const uint4* knew_u = reinterpret_cast<const uint4*>(p.k_new + (size_t)u * D);
    const uint4* vnew_u = reinterpret_cast<const uint4*>(p.v_new + (size_t)u * D);
    const int kept = p.kept_count[bl];
    // query row g of the group as B fragments, bf16
    uint4 qf[NB];
    {
        const uint4* qrow = reinterpret_cast<const uint4*>(p.q + ((size_t)bl * p.H + (size_t)hk * p.G + g) * D);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) qf[kb] = g < p.G ? qrow[kb * 4 + t4] : make_uint4(0, 0, 0, 0);
    }
    const bool appends = rank == 0 && tid < 2 * VPR;         // the CTA that appends the new token's rows
    uint4 fresh_row = make_uint4(0, 0, 0, 0);
    if (appends) fresh_row = (tid < VPR ? knew_u + tid : vnew_u + (tid - VPR))[0];

    // The unit's work is its blocks of 16 decode entries, then its tiles, dealt to the warps of all its CTAs in turn.
    const int n = p.n_old + 1, blocks = (n + 15) / 16;
    const int turn = rank * NW + warp, step = p.nsplit * NW;
    const int first_tile = turn >= blocks ? turn - blocks : (turn - blocks) % step + ((turn - blocks) % step < 0 ? step : 0);
    const int all_tiles = kv4_tiles(p.Mcap);
    const unsigned char* Kt_u = cache.K4 + (size_t)u * all_tiles * F::kKeyTile;
    const unsigned char* Vt_u = cache.V4 + (size_t)u * all_tiles * F::kValueTile;
    const uint32_t wring = smem_u32(ring) + (uint32_t)(warp * NS * Cfg::kStageBytes);
    const auto copy = [&](uint32_t to, const unsigned char* from, auto bytes) {
        constexpr int N = decltype(bytes)::value / 16;       // 16-byte pieces
#pragma unroll
        for (int k = 0; k < (N + 31) / 32; ++k)
            if (k * 32 + 32 <= N || lane < N - k * 32) cp_async16(to + (uint32_t)(k * 512 + lane * 16), from + k * 512 + lane * 16);
    };
    const auto fetch = [&](int tile, int stage) {
        const uint32_t st = wring + (uint32_t)(stage * Cfg::kStageBytes);
        copy(st, Kt_u + (size_t)tile * F::kKeyTile, std::integral_constant<int, F::kKeyTile>());
        if (ATTEND) copy(st + F::kKeyTile, Vt_u + (size_t)tile * F::kValueTile, std::integral_constant<int, F::kValueTile>());
        cp_async_commit();
    };
    // the first tiles are asked for before the kept count is there: tiles below the cap can be read
#pragma unroll
    for (int k = 0; k < NS; ++k) {
        if (first_tile + k * step < all_tiles) fetch(first_tile + k * step, k);
        else cp_async_commit();
    }
    if (FUSED || p.nsplit > 1) cluster_wait();               // all CTAs of the cluster have begun: their memory may be written to
    if (appends)                                             // decode entry n_old
        (tid < VPR ? Kd_u + (size_t)p.n_old * VPR + tid : Vd_u + (size_t)p.n_old * VPR + (tid - VPR))[0] = fresh_row;

    float O[ATTEND ? MT : 1][4];
#pragma unroll
    for (int mt = 0; mt < (ATTEND ? MT : 1); ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c) O[mt][c] = 0.f;
    // of query rows 2*t4 and 2*t4 + 1: the reference (the same in the 8 lanes of a t4), this lane's part of the sum of p, and of w z_v
    float ref[2] = {kUnset, kUnset}, z[2] = {0.f, 0.f}, wz[2] = {0.f, 0.f};
    // lane's logits x[0..1] of key g, x[2..3] of key g + 8, each of rows 2*t4, 2*t4 + 1
    const auto raise = [&](const float (&x)[4]) {            // new references, for all lanes
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float m = fmaxf(x[r], x[2 + r]);
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float up = fmaxf(ref[r], m - kLift);
            const float al = ex2f(ref[r] - up);
            ref[r] = up;
            z[r] *= al;
            wz[r] *= al;
            if (ATTEND)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) O[mt][r] *= al, O[mt][2 + r] *= al;
        }
    };

    // ---- decode entries
#pragma unroll 1
    for (int base = turn * 16; base < n; base += step * 16) {
        const auto row = [&](int j, const uint4* fresh, const uint4* rows) { return j == p.n_old ? fresh : rows + (size_t)j * VPR; };
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        {
            const uint4 *ra = row(base + g, knew_u, Kd_u), *rb = row(base + g + 8, knew_u, Kd_u);
            const bool va = base + g < n, vb = base + g + 8 < n;
            uint4 a[NB], b[NB];
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                a[kb] = load_if(ra + kb * 4 + t4, va);
                b[kb] = load_if(rb + kb * 4 + t4, vb);
            }
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
                const uint32_t f0[4] = {a[kb].x, b[kb].x, a[kb].y, b[kb].y};
                const uint32_t f1[4] = {a[kb].z, b[kb].z, a[kb].w, b[kb].w};
                mma_bf16_16816(c, f0, qf[kb].x, qf[kb].y);
                mma_bf16_16816(c, f1, qf[kb].z, qf[kb].w);
            }
        }
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = base + g + 8 * (i >> 1), r = 2 * t4 + (i & 1);
            x[i] = j < n ? c[i] * p.scale_log2 : SHOTKV_NEG_INF;
            if (j < n && r < p.G) sdec[r * p.Dcap + j] = x[i];
        }
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = x[i] - ref[i & 1];
        if (__any_sync(0xffffffffu, fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])) > kHighest)) {
            raise(x);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = x[i] - ref[i & 1];
        }
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = ex2f(y[i]);
            z[i & 1] += w[i];
        }
        if (ATTEND) {
            // weights as B fragments in three bf16 parts (2^-24), keys in their order on the product's inner side
            uint32_t b0[3], b1[3];
#pragma unroll
            for (int s = 0; s < 3; ++s) {
                const uint32_t lo = pack_bf16(w[0], w[1]), hi = pack_bf16(w[2], w[3]);
                w[0] -= bf16_low(lo), w[1] -= bf16_high(lo), w[2] -= bf16_low(hi), w[3] -= bf16_high(hi);
                b0[s] = transposed(lo), b1[s] = transposed(hi);
            }
            // 16 bytes (8 dimensions) a lane of rows 2*t4, 2*t4 + 1, 2*t4 + 8, 2*t4 + 9: the pairs of a fragment lie in two of them
#pragma unroll
            for (int h = 0; h < NC; ++h) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = base + 2 * t4 + (i & 1) + 8 * (i >> 1);
                    v[i] = load_if(row(j, vnew_u, Vd_u) + h * 8 + g, j < n);
                }
                const uint32_t e[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                          {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a[4] = {__byte_perm(e[0][i], e[1][i], 0x5410), __byte_perm(e[0][i], e[1][i], 0x7632),
                                           __byte_perm(e[2][i], e[3][i], 0x5410), __byte_perm(e[2][i], e[3][i], 0x7632)};
#pragma unroll
                    for (int s = 0; s < 3; ++s) mma_bf16_16816(O[h * 4 + i], a, b0[s], b1[s]);
                }
            }
        }
    }

    // ---- packed rows
    // the queries in f16, the sums of their groups, and what a logit is multiplied by
    float top = 0.f;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
        const uint32_t e[4] = {qf[kb].x, qf[kb].y, qf[kb].z, qf[kb].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(bf16_low(e[i])), fabsf(bf16_high(e[i]))));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int power = min(max((int)(__float_as_uint(top) >> 23), 27), 254) - 141;          // top is about 2^(power + 14)
    const float down = __uint_as_float((uint32_t)(127 - power) << 23);                     // 2^-power
    float qsum[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
        uint32_t e[4] = {qf[kb].x, qf[kb].y, qf[kb].z, qf[kb].w};
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = pack_f16(bf16_low(e[i]) * down, bf16_high(e[i]) * down);
            const float2 v = unpack_f16(e[i]);
            s += v.x + v.y;
        }
        qf[kb] = make_uint4(e[0], e[1], e[2], e[3]);
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        qsum[kb] = s + __shfl_xor_sync(0xffffffffu, s, 2);
    }
    const float scale = p.scale_log2 * __uint_as_float((uint32_t)(127 + power) << 23);
    float qs2[NB][2], scale2[2];                             // of rows 2*t4 and 2*t4 + 1
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        scale2[r] = __shfl_sync(0xffffffffu, scale, 8 * t4 + 4 * r);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) qs2[kb][r] = __shfl_sync(0xffffffffu, qsum[kb], 8 * t4 + 4 * r);
    }

    const int M = min(kept, p.Mcap), tiles = kv4_tiles(M);
    float unit = 1.f;                                        // O and wz are in units of 1 / unit
    bool begun = false;
    int stage = 0;
#pragma unroll 1
    for (int tile = first_tile; tile < tiles; tile += step) {
        cp_async_wait<NS - 1>();
        __syncwarp();
        const unsigned char* st = ring + (size_t)(warp * NS + stage) * Cfg::kStageBytes;
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
            const int key0 = tile * 32 + hb * 16;
            if (hb == 1 && key0 >= M) break;
            const uint4* kc = reinterpret_cast<const uint4*>(st + hb * F::kHalfBytes) + lane;
            const uint32_t* km = reinterpret_cast<const uint32_t*>(st + F::kCodeBytes) + (hb * 16 + g) * NB;
            float x[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t ma[NB], mb[NB];
            if constexpr (NB == 4) {
                const uint4 a = *reinterpret_cast<const uint4*>(km), b = *reinterpret_cast<const uint4*>(km + 8 * NB);
                ma[0] = a.x, ma[1] = a.y, ma[2] = a.z, ma[3] = a.w, mb[0] = b.x, mb[1] = b.y, mb[2] = b.z, mb[3] = b.w;
            } else {
                const uint2 a = *reinterpret_cast<const uint2*>(km), b = *reinterpret_cast<const uint2*>(km + 8 * NB);
                ma[0] = a.x, ma[1] = a.y, mb[0] = b.x, mb[1] = b.y;
            }
#pragma unroll
            for (int h = 0; h < NC; ++h) {
                const uint4 kw = kc[h * 32];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int kb = 2 * h + i;
                    float c[4] = {0.f, 0.f, 0.f, 0.f};
                    uint32_t a[4];
                    codes_f16(i ? kw.z : kw.x, a);
                    mma_f16_16816(c, a, qf[kb].x, qf[kb].y);
                    codes_f16(i ? kw.w : kw.y, a);
                    mma_f16_16816(c, a, qf[kb].z, qf[kb].w);
                    const float sa = bf16_high(ma[kb]), za = bf16_low(ma[kb]), sb = bf16_high(mb[kb]), zb = bf16_low(mb[kb]);
                    x[0] = fmaf(sa, fmaf(za, qs2[kb][0], c[0]), x[0]);
                    x[1] = fmaf(sa, fmaf(za, qs2[kb][1], c[1]), x[1]);
                    x[2] = fmaf(sb, fmaf(zb, qs2[kb][0], c[2]), x[2]);
                    x[3] = fmaf(sb, fmaf(zb, qs2[kb][1], c[3]), x[3]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] *= scale2[i & 1];
            uint32_t va = 0, vb = 0;                         // the values' words of rows g and g + 8
            if (ATTEND) {
                const uint32_t* vm = reinterpret_cast<const uint32_t*>(st + F::kKeyTile + F::kCodeBytes) + hb * 16 + g;
                va = vm[0], vb = vm[8];
            }
            if (key0 + 16 > M) {                             // rows past the count
                if (key0 + g >= M) x[0] = x[1] = SHOTKV_NEG_INF, va = 0;
                if (key0 + g + 8 >= M) x[2] = x[3] = SHOTKV_NEG_INF, vb = 0;
            }
            float y[4], sa = bf16_high(va) * unit, sb = bf16_high(vb) * unit;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = x[i] - ref[i & 1];
            bool out = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])) > kHighest;
            if (ATTEND) out |= !begun || fmaxf(sa, sb) >= 4.f;
            if (__any_sync(0xffffffffu, out)) {
                raise(x);
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = x[i] - ref[i & 1];
                if (ATTEND) {
                    float s = fmaxf(bf16_high(va), bf16_high(vb));
#pragma unroll
                    for (int o = 4; o <= 16; o <<= 1) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, o));
                    const int e = min(max((int)(__float_as_uint(s) >> 23), 67), 250);      // its exponent
                    float next = __uint_as_float((uint32_t)(254 - e) << 23);
                    if (begun) next = fminf(unit, next);
                    const float al = next / unit;
#pragma unroll
                    for (int r = 0; r < 2; ++r) wz[r] *= al;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int c = 0; c < 4; ++c) O[mt][c] *= al;
                    unit = next;
                    begun = true;
                    sa = bf16_high(va) * unit, sb = bf16_high(vb) * unit;
                }
            }
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = ex2f(y[i]);
                z[i & 1] += w[i];
            }
            if (ATTEND) {
                w[0] *= sa, w[1] *= sa, w[2] *= sb, w[3] *= sb;
                const float za = bf16_low(va), zb = bf16_low(vb);
                wz[0] = fmaf(w[0], za, fmaf(w[2], zb, wz[0]));
                wz[1] = fmaf(w[1], za, fmaf(w[3], zb, wz[1]));
                const uint32_t h0 = pack_f16(w[0], w[1]), h1 = pack_f16(w[2], w[3]);
                const float2 f0 = unpack_f16(h0), f1 = unpack_f16(h1);
                const uint32_t bh0 = transposed(h0), bh1 = transposed(h1);
                const uint32_t bl0 = transposed(pack_f16(w[0] - f0.x, w[1] - f0.y)), bl1 = transposed(pack_f16(w[2] - f1.x, w[3] - f1.y));
                const uint4* vc = reinterpret_cast<const uint4*>(st + F::kKeyTile + hb * F::kHalfBytes) + lane;
#pragma unroll
                for (int h = 0; h < NC; ++h) {
                    const uint4 vw = vc[h * 32];
                    const uint32_t e[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t a[4];
                        codes_f16(e[i], a);
                        mma_f16_16816(O[h * 4 + i], a, bh0, bh1);
                        mma_f16_16816(O[h * 4 + i], a, bl0, bl1);
                    }
                }
            }
        }
        __syncwarp();                                       // every lane has read the stage the next copy overwrites
        if (tile + NS * step < tiles) fetch(tile + NS * step, stage);
        else cp_async_commit();
        stage = stage + 1 == NS ? 0 : stage + 1;
    }
    cp_async_wait<0>();

    // ---- the warp's rows
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int o = 4; o <= 16; o <<= 1) {
            z[r] += __shfl_xor_sync(0xffffffffu, z[r], o);
            if (ATTEND) wz[r] += __shfl_xor_sync(0xffffffffu, wz[r], o);
        }
    if (g == 0)
#pragma unroll
        for (int r = 0; r < 2; ++r) sred[warp * 8 + 2 * t4 + r] = make_float2(z[r] == 0.f ? SHOTKV_NEG_INF : ref[r], z[r]);
    __syncwarp();                                           // all lanes are done with the warp's ring: its outputs take its place
    constexpr int kPitch = NS * Cfg::kStageBytes / 4;       // floats
    float* sO = reinterpret_cast<float*>(ring);
    if (ATTEND) {
        const float back = 1.f / unit;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int h = 0; h < NC; ++h) {
                float* o = sO + warp * kPitch + (2 * t4 + r) * kOutPitch<D> + h * 64 + g * 8;
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[2 * i] = (O[h * 4 + i][r] + wz[r]) * back, v[2 * i + 1] = (O[h * 4 + i][2 + r] + wz[r]) * back;
                *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
    }
    __syncthreads();
    if constexpr (ATTEND) {
        finish_attend<D, NW, FUSED>(p, f, UnitPart{u, bl, hk, rank, first_cta, ctas}, qs, end, sred, sdec, stab, sin, arrived, sO, kPitch, turn * 16);
    } else {
        bool ok = true;
        if (p.nsplit > 1) {
            if (tid < 8 * p.nsplit) {                       // every CTA's rows to every CTA
                float fac[NW];
                send(stab + rank * 8 + (tid & 7), first_cta + (tid >> 3), arrived, row_of_cta(sred, tid & 7, fac));
            }
            ok = await_messages(arrived, p.err, p.wait_cycles);
        }
        float rm, riz;
        row_of_unit(p.nsplit > 1 ? stab : sred, p.nsplit > 1 ? p.nsplit : NW, rm, riz);
        const bool whole = p.nsplit == 1;
        entry_weights(sdec, p.Dcap, p.G, rm, riz, whole ? warp * 32 : turn * 16, n, whole ? NW * 32 : step * 16, whole ? 32 : 16, [&](int j, float s) {
            if (FUSED) fused_send(end, f, hk, j, s, ctas);
            else p.partial[(size_t)u * p.Dcap + j] = s;
        });
        const bool all = !FUSED || fused_finish<D, NW * 32>(end, f, bl, first_cta + rank, ctas, p);
        if (!(ok && all)) outlive_messages(ok ? nullptr : arrived, all ? nullptr : end.arrived, p.err, p.wait_cycles);
    }
}

}  // namespace shotkv
