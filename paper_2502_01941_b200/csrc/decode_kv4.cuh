// The decode steps over a prompt's cache held in 4 bits (kv4.cuh).
#pragma once
#include <type_traits>

#include "decode.cuh"
#include "kv4.cuh"
#include "ring.cuh"
#include "score_tc.cuh"

namespace shotkv {

// D(16x8,f32) += A(16x16,f16,row) * B(16x8,f16,col)
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same with nothing to add to.  (With zeros in the accumulator beforehand they were 60 moves a tile.)
__device__ __forceinline__ void mma_f16_16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
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

// `bytes` (a multiple of 16) from global to this CTA's shared memory; they are counted on the barrier when they have landed.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
                 "r"(bar)
                 : "memory");
}

__device__ __forceinline__ uint64_t sub_pairs(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// Of each of two matrices of 8 keys, columns 0 .. 3 are to be one number of every key and columns 4 .. 7 another.  The lanes of columns
// 0 .. 3 have both numbers of the first matrix's keys, those of columns 4 .. 7 (`second`) of the other's: what each contributes to them.
__device__ __forceinline__ void halves_of_columns(uint32_t one, uint32_t another, bool second, uint32_t& matrix0, uint32_t& matrix1) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, second ? one : another, 2);
    matrix0 = second ? other : one;
    matrix1 = second ? another : other;
}

struct PackedCache {
    const unsigned char *K4, *V4;            // [U][tiles][Kv4 tile]
};

template <int D, bool ATTEND, bool PAIRED>
struct StepKv4 {
    static constexpr int kWarps = 4;
    static constexpr int kStages = ATTEND ? 2 : 3;         // tiles in a warp's ring
    static constexpr int kStageBytes = Kv4<D>::kKeyTile + (ATTEND ? Kv4<D>::kValueTile : 0);
    static constexpr int kRingBytes = kWarps * kStages * kStageBytes;
    static constexpr int kBarBytes = kWarps * kStages * 8;
    // CTAs on an SM that the registers are meant for.  (8 sequences x 32 layers, us a step.  d = 128, attention output: 4 and 5 CTAs the
    // same, 5 with spilled registers.  d = 64: 700 rows 4 | 5 CTAs 53.6 | 47.7, but eight query rows 133.5 | 135.2.  Scores,
    // d = 128 5 | 6 99.8 | 101.1, of 4 sequences 59.5 | 57.2; d = 64 6 | 8 60.6 | 64.9.)
    static constexpr int ctas(bool fused) { return fused ? 3 : !ATTEND ? 6 : D == 64 && PAIRED ? 5 : 4; }
    static constexpr int kQueryBytes = (PAIRED ? 2 : 1) * 8 * D * 2 + (D / 32) * 8 * 4;    // operands of 8 columns in f16, the rows' groups' sums
    static_assert(!ATTEND || 8 * kOutPitch<D> * 4 <= kStages * kStageBytes, "a warp's outputs take the place of its ring");
};
template <int D, bool ATTEND, bool PAIRED>
__host__ __device__ constexpr size_t kv4_smem_bytes(int G, int Dcap, int nsplit) {
    const size_t shares = nsplit > 1 ? (size_t)nsplit * (16 + (ATTEND ? (G * D / 4 / nsplit + 1) * 4 : 0)) : 0;
    using Cfg = StepKv4<D, ATTEND, PAIRED>;
    return Cfg::kRingBytes + Cfg::kBarBytes + Cfg::kQueryBytes + 16 + ((size_t)Cfg::kWarps * 16 + ((size_t)G * Dcap + 3) / 4 * 4 + shares) * 4;
}

// decode_score_kernel's and (ATTEND) decode_attend_kernel's step over packed prefill rows.  A warp takes decode entries,
// which are bf16, 16 at a time straight from global memory, and packed rows a tile of 32 at a time through its ring.
//
// Both products have the keys, or the values' dimensions, on the 16-row side, so that a packed word is an operand's
// fragment but for the conversion, and the group's (up to 8) query rows on the side of 8:
//   S[16 keys x 8 rows] = (c + 8) . q, one chain of products for every group of 32 dimensions, in f16: codes are whole numbers (as
//     f16 subnormals: nothing but masks and a shift), and a query row, bf16, is multiplied by the power of two that takes its
//     largest element to [2^14, 2^15), which leaves elements down to 2^-31 of it exact.  A logit is the sum over groups of
//     s (S + (z - 8) times the sum of q's 32 elements).
//   O^T[16 dims x 8 rows] += c^T . w^T with w = p s_v, p = 2^(logit - reference): the accumulator of S, transposed 8 by 8, is
//     the other operand, an f16 pair (high part and remainder: 2^-22 of w, or half of f16's least step, 2^-25).  z is added once a
//     row: sum of w z_v.
// PAIRED, for groups of up to four rows: the columns 4 .. 7 are the same rows again.  The remainders are in these columns of the one
// operand whose columns 0 .. 3 are the high parts, so that one product does for both, and the lanes of columns 0 .. 3 have the
// logits of one half of a tile, those of columns 4 .. 7 of the other.  (8 sequences x 32 layers, 3,276 rows, 145
// entries, captured: four query rows 186 us a step, eight, each half and part with products of its own, 219.)
//
// f16 ends at 65504, so both factors are kept in range by references that change seldom: a row's reference is 2^10 below its
// maximum when it was last set and is set again by a tile whose p would exceed 2^13, and the values' scales are multiplied by a
// power of two that takes the largest of the first tile to [1, 2) and is set again by a tile more than half of whose scales it leaves
// outside [2^-8, 4); a tile's rows that are outside are added by themselves.  So a weight is off by no
// more than 2^-27 of the row's largest (2^-35 where the scales are alike), whatever the others' values are.  One vote a tile
// decides that nothing of this has happened.  (8 sequences x 32 layers, 3,276 rows, one value in 1,000, in 32, in 8 of 2^10 or 2^-10
// of the others' scale: 189, 250, 377 us.)  A matrix unit cuts off what does not fit its sums, always towards zero, so a tile's
// products are summed for themselves and then added: one sum for all of a warp's 26 tiles left the outputs 4.2e-6 off in the
// 2-norm, so they are 5.5e-7 off (elementary operations in 32 bits: 9.2e-7).  Scores are 2.6e-7 off (1.5e-7): s (c + 8) . q and s (z - 8)
// times the sum of q are rounded apart.
//
// What bounds it: bytes from HBM where calls are far apart (that step reads 1.09 GB: 178 us with kept counts that differ, 6.1 TB/s), and
// the power cap where they follow one another for long (198 to 210 us from GPU to GPU, at 1.6 to 1.7 GHz): about 480 instructions a tile, half of them
// conversions and the groups' scales, at 0.6 to 0.7 a cycle and scheduler.  So what was saved is instructions (780 at first): bulk
// copies that one lane asks for, no accumulator set to zero, constants that stay in registers, sums of two rows at a time.  More
// CTAs on an SM, or one tile's values computed beside the next one's keys, gained nothing.  Scores alone read half: 96 us, 6.0 TB/s.
template <int D, bool ATTEND, bool FUSED, bool PAIRED>
__global__ void __launch_bounds__(StepKv4<D, ATTEND, PAIRED>::kWarps * 32, StepKv4<D, ATTEND, PAIRED>::ctas(FUSED))
decode_kv4_kernel(const DecodeParams p, const DecodeFinishParams f, const PackedCache cache) {
    using Cfg = StepKv4<D, ATTEND, PAIRED>;
    using F = Kv4<D>;
    constexpr int NB = D / 32, NC = D / 64, VPR = D / 8, MT = D / 16;
    constexpr int NW = Cfg::kWarps, NS = Cfg::kStages;
    constexpr float kLift = 10.f, kHighest = 8192.f, kUnset = -3.402823466e38f, kCoarse = 0x1p22f;
    extern __shared__ __align__(128) unsigned char dsm[];
    unsigned char* ring = dsm;                               // [NW][NS][keys | values]; later each warp's outputs
    uint4* sq = reinterpret_cast<uint4*>(ring + Cfg::kRingBytes + Cfg::kBarBytes);   // [1, PAIRED 2][NB][32 lanes] the queries as B fragments, f16
    float* sqsum = reinterpret_cast<float*>(sq + (PAIRED ? 2 : 1) * NB * 32);                   // [NB][8 rows] their groups' sums
    float2* sred = reinterpret_cast<float2*>(ring + Cfg::kRingBytes + Cfg::kBarBytes + Cfg::kQueryBytes + 16);   // [NW warps][8 rows]  (m, z)
    float* sdec = reinterpret_cast<float*>(sred + NW * 8);   // [G][Dcap]  logits of the decode entries
    float2* stab = reinterpret_cast<float2*>(sdec + ((p.G * p.Dcap + 3) & ~3));
    float4* sin = reinterpret_cast<float4*>(stab + p.nsplit * 8);
    unsigned long long* arrived = reinterpret_cast<unsigned long long*>(sred) - 1;

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;     // (so that the warp's are uniform)
    const int g = lane >> 2, t4 = lane & 3;
    const int u = blockIdx.x / p.nsplit, rank = blockIdx.x - u * p.nsplit;
    const QuadShare qs = quads_of<D>(p.G, p.nsplit, rank);
    const int bl = u / p.Hkv, hk = u - bl * p.Hkv;
    const int first_cta = FUSED ? hk * p.nsplit : 0, ctas = p.Hkv * p.nsplit;   // in the cluster: the unit's first; FUSED: all
    FusedEnd end{};
    if (FUSED) end = fused_end_at(dsm + kv4_smem_bytes<D, ATTEND, PAIRED>(p.G, p.Dcap, p.nsplit), f);
    unsigned long long* bars = reinterpret_cast<unsigned long long*>(ring + Cfg::kRingBytes) + warp * NS;   // this warp's stages'
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < NS; ++k) tc::mbar_init(smem_u32(bars + k), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
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
    // query rows as B fragments: columns 0 .. 7 are the group's rows, or (PAIRED) its up to four rows twice.  This lane's column of
    // an operand is g, and of an accumulator 2*t4 and 2*t4 + 1, which are rows r0 and r0 + 1.
    const int g_row = PAIRED ? g & 3 : g, r0 = PAIRED ? (2 * t4) & 3 : 2 * t4;
    const bool second = PAIRED && t4 >= 2;                   // the columns of the weights' remainders
    // Of 16 decode entries in an accumulator a lane has g and g + 8, and both in both columns of a row where there are two: it
    // goes on with the first or the second of them then.
    constexpr int KL = PAIRED ? 1 : 2;
    const auto key_of = [&](int k) { return g + (k || second ? 8 : 0); };
    const uint4* qrow = reinterpret_cast<const uint4*>(p.q + ((size_t)bl * p.H + (size_t)hk * p.G + g_row) * D);
    uint4 qf[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) qf[kb] = load_if(qrow + kb * 4 + t4, g_row < p.G);
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
    const unsigned char* mine = ring + warp * NS * Cfg::kStageBytes;         // this warp's ring
    // One lane asks for a tile, in one copy of its keys and one of its values: as 16-byte copies, ten a lane, these and
    // their addresses were a tenth of the loop's instructions.
    const auto fetch = [&](int tile, int stage) {
        if (lane != 0) return;
        const uint32_t st = smem_u32(mine) + (uint32_t)(stage * Cfg::kStageBytes), bar = smem_u32(bars + stage);
        tc::mbar_expect_tx(bar, Cfg::kStageBytes);
        bulk_load(st, Kt_u + (size_t)tile * F::kKeyTile, F::kKeyTile, bar);
        if (ATTEND) bulk_load(st + F::kKeyTile, Vt_u + (size_t)tile * F::kValueTile, F::kValueTile, bar);
    };
    // The first are asked for before the kept count is there: tiles below the cap can be read.
    TileRing<NS> ahead(first_tile, step);
    ahead.ask(all_tiles, fetch);
    if (FUSED || p.nsplit > 1) cluster_wait();               // all CTAs of the cluster have begun: their memory may be written to
    if (appends)                                             // decode entry n_old
        (tid < VPR ? Kd_u + (size_t)p.n_old * VPR + tid : Vd_u + (size_t)p.n_old * VPR + (tid - VPR))[0] = fresh_row;

    // The queries in f16, the sums of their groups, and what a logit is multiplied by.  They lie in shared memory: in
    // registers they would take a CTA from the SM.
    float scale2[2];                                         // of rows 2*t4 and 2*t4 + 1
    {
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
        // of a query row beyond 2^115, whose factor is beyond float32, its negative without 2^24
        float scale = p.scale_log2 * __uint_as_float((uint32_t)(127 + power) << 23);
        scale *= power > 100 ? -1.f : 0x1p24f;
#pragma unroll
        for (int r = 0; r < 2; ++r) scale2[r] = __shfl_sync(0xffffffffu, scale, 8 * t4 + 4 * r);
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
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            if (warp == kb) {
                // paired, an operand for each half of a tile: the rows in columns 0 .. 3, and in columns 4 .. 7, the others zeros
                const uint4 q = make_uint4(e[0], e[1], e[2], e[3]), none = make_uint4(0, 0, 0, 0);
                sq[kb * 32 + lane] = PAIRED && g >= 4 ? none : q;
                if (PAIRED) sq[(NB + kb) * 32 + lane] = g >= 4 ? q : none;
                if (t4 == 0) sqsum[kb * 8 + g] = s * 0x1p-24f;
            }
        }
    }
    static_assert(NB <= NW, "a warp writes one block of the queries");
    __syncthreads();

    float O[ATTEND ? MT : 1][4];
#pragma unroll
    for (int mt = 0; mt < (ATTEND ? MT : 1); ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c) O[mt][c] = 0.f;
    // of query rows 2*t4 and 2*t4 + 1: the reference (the same in the 8 lanes of a t4), this lane's part of the sum of p, and of w z_v
    float ref[2] = {kUnset, kUnset}, z[2] = {0.f, 0.f}, wz[2] = {0.f, 0.f};
    constexpr int kFirstLane = PAIRED ? 2 : 4;               // lanes a row's keys are spread over: those of one t4, or of t4 and t4 ^ 2
    // What a tile's weights may be.  From 2^22 on a logit's own rounding counts: as a multiply-add its weight would be that of the exact
    // product, apart from the reference by up to half a step of 32 bits.  So a warp that has met one so large, or a query row whose
    // factor is in two parts, looks at every tile again, where logits are rounded before the reference is subtracted, as the
    // entries' are.
    float highest = __any_sync(0xffffffffu, fminf(scale2[0], scale2[1]) < 0.f) ? -1.f : kHighest;
    const auto raise = [&](const float (&high)[2]) {         // new references, from all lanes' greatest logits
        bool coarse = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float m = high[r];
#pragma unroll
            for (int o = kFirstLane; o <= 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            // (a logit of 2^27 or more has steps of 16 and more: it is its own reference)
            const float up = fmaxf(ref[r], fabsf(m) < 0x1p27f ? m - kLift : m);
            const float al = ex2f(ref[r] - up);
            ref[r] = up;
            coarse |= up != kUnset && fabsf(up) >= kCoarse;
            z[r] *= al;
            wz[r] *= al;
            if (ATTEND)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) O[mt][r] *= al, O[mt][2 + r] *= al;
        }
        if (__any_sync(0xffffffffu, coarse)) highest = -1.f;
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
                const uint4 q = load_if(qrow + kb * 4 + t4, g_row < p.G);
                mma_bf16_16816(c, f0, q.x, q.y);
                mma_bf16_16816(c, f1, q.z, q.w);
            }
        }
        float x[2 * KL];                                     // of this lane's keys, each its two rows
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i) {
            const int j = base + key_of(i >> 1), r = r0 + (i & 1);
            x[i] = j < n ? (second ? c[2 + (i & 1)] : c[i]) * p.scale_log2 : SHOTKV_NEG_INF;
            if (j < n && r < p.G) sdec[r * p.Dcap + j] = x[i];
        }
        float w[2 * KL], most = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i) most = fmaxf(most, w[i] = ex2f(x[i] - ref[i & 1]));
        if (__any_sync(0xffffffffu, most > kHighest)) {
            const float high[2] = {fmaxf(x[0], x[2 * KL - 2]), fmaxf(x[1], x[2 * KL - 1])};
            raise(high);
#pragma unroll
            for (int i = 0; i < 2 * KL; ++i) w[i] = ex2f(x[i] - ref[i & 1]);
        }
#pragma unroll
        for (int i = 0; i < 2 * KL; ++i) z[i & 1] += w[i];
        if (ATTEND) {
            // weights as B fragments in three bf16 parts (2^-24), keys in their order on the product's inner side; paired, the
            // first two are the columns of one fragment
            constexpr int PARTS = PAIRED ? 2 : 3;
            uint32_t b0[3], b1[3];
#pragma unroll
            for (int s = 0; s < 3; ++s)
#pragma unroll
                for (int k = 0; k < KL; ++k) {
                    uint32_t& b = k ? b1[s] : b0[s];
                    b = pack_bf16(w[2 * k], w[2 * k + 1]);
                    w[2 * k] -= bf16_low(b), w[2 * k + 1] -= bf16_high(b);
                }
            if constexpr (PAIRED) {
                const uint32_t l = b0[2], other = __shfl_xor_sync(0xffffffffu, l, 2);
                halves_of_columns(b0[0], b0[1], second, b0[0], b1[0]);
                b0[1] = second ? 0u : l, b1[1] = second ? 0u : other;
            }
#pragma unroll
            for (int s = 0; s < PARTS; ++s) b0[s] = transposed(b0[s]), b1[s] = transposed(b1[s]);
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
                    for (int s = 0; s < PARTS; ++s) mma_bf16_16816(O[h * 4 + i], a, b0[s], b1[s]);
                }
            }
        }
    }

    // ---- packed rows
    const int M = min(kept, p.Mcap), tiles = kv4_tiles(M);
    // codes_subnormal has c + 8 multiplied, and of key g + 8 sixteen times that
    const float scales[2][2] = {{scale2[0], scale2[1]}, {scale2[0] * 0.0625f, scale2[1] * 0.0625f}};
    // Paired, the products of both halves of a tile add up in one accumulator, the first half's in columns 0 .. 3: a lane has keys g
    // and g + 8 of one of them (all columns with both halves' keys, one of each two chosen: 212 us a step
    // at the power cap where this takes 208).
    constexpr int HALVES = PAIRED ? 1 : 2;                   // of a tile, that a lane has keys of
    const auto half_of = [&](int h) { return PAIRED ? (int)second : h; };
    // A tile's weights times scales are in units of back = 1 / unit; the first tile of all sets them.
    float unit = 0x1p100f, back = 0x1p-100f;
    if (ATTEND)                                              // odd dimensions' are sixteen times as much from here on
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) O[mt][2] *= 16.f, O[mt][3] *= 16.f;
    // in registers that the compiler cannot make anew for each use
    Under under = codes_under();
    under.k1024 |= (uint32_t)p.nsplit >> 31, under.k1032 |= (uint32_t)p.nsplit >> 31;
    // Scales of 2^-8 to 4 in these units, as a value's word less the least of them: 0 to kSpan - 1.
    constexpr uint32_t kSpan = 10u << 23;
    const auto above = [&](uint32_t word) { return word - (__float_as_uint(back) - (8u << 23)); };
    // The value in lane `src` of those that hold the first of the query rows (its half of the tile h, where a lane has both; row g + 8 k
    // of it) times its weights, in plain multiply-adds.
    const auto add_row = [&](const unsigned char* st, int src, int h, int k, float w0, float w1, uint32_t word) {
        const int r = src >> 2, half = PAIRED ? src >> 1 & 1 : h, from = src + (PAIRED ? t4 & 1 : t4);
        w0 = __shfl_sync(0xffffffffu, w0, from), w1 = __shfl_sync(0xffffffffu, w1, from);
        word = __shfl_sync(0xffffffffu, word, src);
        const float s = bf16_high(word), z8 = bf16_low(word) - 8.f;
        const uint4* vc = reinterpret_cast<const uint4*>(st + F::kKeyTile + half * F::kHalfBytes) + 4 * g + (r >> 1);
        if (second) return;                                  // its columns are the remainders of the same rows
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 v4 = vc[c * 32];
            const uint32_t v[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = (float)(v[i] >> (4 * (e + 2 * k) + 16 * (r & 1)) & 15u) + z8, y = s * (e ? 16.f * x : x);
                    O[c * 4 + i][2 * e] = fmaf(w0, y, O[c * 4 + i][2 * e]);
                    O[c * 4 + i][2 * e + 1] = fmaf(w1, y, O[c * 4 + i][2 * e + 1]);
                }
        }
    };
    // The same answer in all lanes; `limit` cycles at most.
    const auto landed = [&](int stage, uint32_t parity, long long limit) {
        bool there = tc::mbar_try(smem_u32(bars + stage), parity);
        if (__all_sync(0xffffffffu, there)) return true;
        there = there || await_messages(bars + stage, p.err, limit, parity);
        return (bool)__all_sync(0xffffffffu, there);
    };
#pragma unroll 1
    while (ahead.tile < tiles) {
        if (!landed(ahead.stage, ahead.parity, p.wait_cycles)) break;     // the warp goes on with what it has
        const int tile = ahead.tile;
        const unsigned char* st = mine + ahead.stage * Cfg::kStageBytes;
        // of this lane's halves, logits of keys g (x[.][0..1], still to be scaled) and g + 8 (x[.][2..3]), and the values' words
        float x[HALVES][4] = {};
        uint32_t m[HALVES][2][NB], vw[HALVES][2];
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int row = half_of(h) * 16 + g + 8 * k;
                const uint32_t* km = reinterpret_cast<const uint32_t*>(st + F::kCodeBytes) + row * NB;
                if constexpr (NB == 4) {
                    const uint4 a = *reinterpret_cast<const uint4*>(km);
                    m[h][k][0] = a.x, m[h][k][1] = a.y, m[h][k][2] = a.z, m[h][k][3] = a.w;
                } else {
                    const uint2 a = *reinterpret_cast<const uint2*>(km);
                    m[h][k][0] = a.x, m[h][k][1] = a.y;
                }
                if (ATTEND) vw[h][k] = reinterpret_cast<const uint32_t*>(st + F::kKeyTile + F::kCodeBytes)[row];
            }
        const uint4* kc = reinterpret_cast<const uint4*>(st) + lane;
#pragma unroll
        for (int c64 = 0; c64 < NC; ++c64) {
            const uint4 k0 = kc[c64 * 32], k1 = kc[F::kHalfBytes / 16 + c64 * 32];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int kb = 2 * c64 + i;
                const uint4 q = sq[kb * 32 + lane];
                const float2 qsum = *reinterpret_cast<const float2*>(sqsum + kb * 8 + r0);
                float c[2][4];
                uint32_t a[4];
                codes_subnormal(i ? k0.z : k0.x, a);
                mma_f16_16816_first(c[0], a, q.x, q.y);
                codes_subnormal(i ? k0.w : k0.y, a);
                mma_f16_16816(c[0], a, q.z, q.w);
                if constexpr (PAIRED) {
                    const uint4 r = sq[(NB + kb) * 32 + lane];
                    codes_subnormal(i ? k1.z : k1.x, a);
                    mma_f16_16816(c[0], a, r.x, r.y);
                    codes_subnormal(i ? k1.w : k1.y, a);
                    mma_f16_16816(c[0], a, r.z, r.w);
                } else {
                    codes_subnormal(i ? k1.z : k1.x, a);
                    mma_f16_16816_first(c[1], a, q.x, q.y);
                    codes_subnormal(i ? k1.w : k1.y, a);
                    mma_f16_16816(c[1], a, q.z, q.w);
                }
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float s = bf16_high(m[h][k][kb]), z8 = bf16_low(m[h][k][kb]), zs = k ? fmaf(z8, 16.f, -128.f) : z8 - 8.f;
                        x[h][2 * k] = fmaf(s, fmaf(zs, qsum.x, c[h][2 * k]), x[h][2 * k]);
                        x[h][2 * k + 1] = fmaf(s, fmaf(zs, qsum.y, c[h][2 * k + 1]), x[h][2 * k + 1]);
                    }
            }
        }
        if (tile * 32 + 32 > M)                              // rows past the count
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (tile * 32 + half_of(h) * 16 + g + 8 * k >= M) x[h][2 * k] = x[h][2 * k + 1] = SHOTKV_NEG_INF, vw[h][k] = __float_as_uint(back);
        // weights relative to the references, which are set again where one is out of range
        float w[HALVES][4];
        {
            const uint64_t down = tc::pack2(-ref[0], -ref[1]);
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float y0, y1;
                    tc::unpack2(tc::ffma2(tc::pack2(x[h][2 * k], x[h][2 * k + 1]), tc::pack2(scales[k][0], scales[k][1]), down), y0, y1);
                    w[h][2 * k] = ex2f(y0), w[h][2 * k + 1] = ex2f(y1);
                }
        }
        {
            float most = 0.f;
            uint32_t far = 0;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                most = fmaxf(most, fmaxf(fmaxf(w[h][0], w[h][1]), fmaxf(w[h][2], w[h][3])));
                if (ATTEND) far = max(far, max(above(vw[h][0]), above(vw[h][1])));
            }
            if (__any_sync(0xffffffffu, most > highest || far >= kSpan)) {
                float high[2] = {SHOTKV_NEG_INF, SHOTKV_NEG_INF};
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) {
                    float& v = x[i / 4][i % 4];
                    const float scale = scales[i / 2 % 2][i & 1];
                    v = __fmul_rn(v, scale) * (scale < 0.f ? -0x1p24f : 1.f);
                    high[i & 1] = fmaxf(high[i & 1], v);
                }
                raise(high);
#pragma unroll
                for (int i = 0; i < 4 * HALVES; ++i) w[i / 4][i % 4] = ex2f(x[i / 4][i % 4] - ref[i & 1]);
                if (ATTEND && __any_sync(0xffffffffu, far >= kSpan)) {
                    // Other units where these do for less than half of the tile's rows: those of the greatest scale, or if they
                    // do not do either of the greatest below them, and so on.  Rows that the units do not do for are added by themselves.
                    constexpr uint32_t kOnce = PAIRED ? 0x55555555u : 0x11111111u;        // of the lanes with a row's word one
#pragma unroll
                    for (int i = 0; i < 2 * HALVES; ++i)
                        if (tile * 32 + half_of(i / 2) * 16 + g + 8 * (i % 2) >= M) vw[i / 2][i % 2] = 0;
                    uint32_t below = 0x7f800000u;            // (so of the scales that are numbers)
#pragma unroll 1
                    for (;;) {
                        int fit = 0;
#pragma unroll
                        for (int i = 0; i < 2 * HALVES; ++i)
                            fit += __popc(__ballot_sync(0xffffffffu, above(vw[i / 2][i % 2]) < kSpan) & kOnce);
                        if (2 * fit >= min(32, M - tile * 32)) break;
                        float s = 0.f;
#pragma unroll
                        for (int i = 0; i < 2 * HALVES; ++i)
                            s = fmaxf(s, vw[i / 2][i % 2] < below ? bf16_high(vw[i / 2][i % 2]) : 0.f);
#pragma unroll
                        for (int o = kFirstLane; o <= 16; o <<= 1) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, o));
                        if (!(s >= 0x1p-100f)) break;        // none, or what was never packed: every turn goes lower, to here
                        const uint32_t e = min(__float_as_uint(s) >> 23, 250u);            // its exponent, 27 or more
                        unit = __uint_as_float((254 - e) << 23), back = __uint_as_float(e << 23);
                        below = (e - 8) << 23;
                    }
                    const auto apart = [&](uint32_t word) { return word != 0 && above(word) >= kSpan; };
                    bool some = false;
#pragma unroll
                    for (int i = 0; i < 2 * HALVES; ++i) some |= apart(vw[i / 2][i % 2]);
                    if (__any_sync(0xffffffffu, some))
#pragma unroll
                        for (int h = 0; h < HALVES; ++h)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const bool alone = apart(vw[h][k]);
                                uint32_t lanes = __ballot_sync(0xffffffffu, alone) & kOnce;
#pragma unroll 1
                                for (; lanes; lanes &= lanes - 1) add_row(st, __ffs(lanes) - 1, h, k, w[h][2 * k], w[h][2 * k + 1], vw[h][k]);
                                if (alone) vw[h][k] = 0;
                            }
                }
            }
        }
        // their sums, and with the values' scales (ATTEND) they are B fragments of the halves' eights of keys: high parts and remainders
        uint32_t wh[2][2], wl[2][2];
        uint64_t zz = tc::pack2(z[0], z[1]);
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float w0 = w[h][2 * k], w1 = w[h][2 * k + 1];
                zz = tc::fadd2(zz, tc::pack2(w0, w1));
                if (ATTEND) {
                    const float s = bf16_high(vw[h][k]), sz = s * bf16_low(vw[h][k]), su = s * unit;
                    wz[0] = fmaf(w0, sz, wz[0]);
                    wz[1] = fmaf(w1, sz, wz[1]);
                    w0 *= su, w1 *= su;
                    const uint32_t hi = pack_f16(w0, w1);
                    const float2 f = unpack_f16(hi);
                    float rest[2];
                    tc::unpack2(sub_pairs(tc::pack2(w0, w1), tc::pack2(f.x, f.y)), rest[0], rest[1]);
                    const uint32_t lo = pack_f16(rest[0], rest[1]);
                    if constexpr (PAIRED) {
                        halves_of_columns(hi, lo, second, wh[0][k], wh[1][k]);
                        wh[0][k] = transposed(wh[0][k]), wh[1][k] = transposed(wh[1][k]);
                    } else {
                        wh[h][k] = transposed(hi), wl[h][k] = transposed(lo);
                    }
                }
            }
        tc::unpack2(zz, z[0], z[1]);
        if (ATTEND) {
            const uint4* vc = reinterpret_cast<const uint4*>(st + F::kKeyTile) + lane;
            const uint64_t back2 = tc::pack2(back, back);
#pragma unroll
            for (int h = 0; h < NC; ++h) {
                const uint4 v0 = vc[h * 32], v1 = vc[F::kHalfBytes / 16 + h * 32];
                const uint32_t e0[4] = {v0.x, v0.y, v0.z, v0.w}, e1[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float c[4];
                    uint32_t a[4];
                    codes_f16(e0[i], under, a);
                    if (PAIRED) mma_f16_16816_first(c, a, wh[0][0], wh[0][1]);
                    else mma_f16_16816_first(c, a, wl[0][0], wl[0][1]), mma_f16_16816(c, a, wh[0][0], wh[0][1]);
                    codes_f16(e1[i], under, a);
                    if (!PAIRED) mma_f16_16816(c, a, wl[1][0], wl[1][1]);
                    mma_f16_16816(c, a, wh[1][0], wh[1][1]);
                    float(&o)[4] = O[h * 4 + i];
                    tc::unpack2(tc::ffma2(tc::pack2(c[0], c[1]), back2, tc::pack2(o[0], o[1])), o[0], o[1]);
                    tc::unpack2(tc::ffma2(tc::pack2(c[2], c[3]), back2, tc::pack2(o[2], o[3])), o[2], o[3]);
                }
            }
        }
        __syncwarp();                                       // every lane has read the stage the next copy overwrites
        ahead.next(tiles, fetch);
    }
    ahead.land(all_tiles, tiles, landed);

    // ---- the warp's rows
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int o = kFirstLane; o <= 16; o <<= 1) {
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
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int h = 0; h < NC; ++h) {
                float* o = sO + warp * kPitch + (r0 + r) * kOutPitch<D> + h * 64 + g * 8;
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = O[h * 4 + i][2 * e + r];
                        if (PAIRED) x += __shfl_xor_sync(0xffffffffu, x, 2);
                        v[2 * i + e] = e ? fmaf(x, 0.0625f, wz[r]) : x + wz[r];
                    }
                if (!second) {
                    *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
    }
    __syncthreads();
    if constexpr (ATTEND) {
        finish_attend<D, NW, FUSED>(p, f, UnitPart{u, bl, hk, rank, first_cta, ctas}, qs, end, sred, sdec, stab, sin, arrived, sO, kPitch,
                                        turn * 16, 0, n);
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
        if (!(ok && all)) outlive_messages(ok ? nullptr : arrived, all ? nullptr : end.arrived, p.err);
    }
}

}  // namespace shotkv
