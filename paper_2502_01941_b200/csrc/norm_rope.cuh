// From a layer's projection to the tensors that the other calls take: queries and keys normed per head and rotated by
// position, values as they are, each written in its place.
#pragma once
#include "common.cuh"
#include "score_tc.cuh"

namespace shotkv {

struct NormRopeParams {
    const __nv_bfloat16 *q, *k, *v;          // [B][rows][heads][D], rows and prompts `*_row` and `*_prompt` elements apart
    long long q_row, k_row, v_row, q_prompt, k_prompt, v_prompt;
    const __nv_bfloat16 *q_weight, *k_weight;    // [D], or NULL: not normed
    const float2* table;                     // [table_rows][rot / 2]  (cos, sin)
    const int* positions;                    // [B][rows], or NULL: first + row
    __nv_bfloat16 *Qwin, *K, *V;             // [B][L][H][W][D], [B][L][Hkv][N][D] twice
    __nv_bfloat16* q_out;                    // [B][rows][H][D], or NULL
    int B, L, H, Hkv, N, W, layer, first, rows, rot, interleaved, table_rows;
    int q_first;                             // first row whose queries are wanted
    float eps;
    // dealing rows to warps: pieces of 16 bytes a lane that a row's heads take, cut into sections of so many; CTAs that have
    // keys and values, before those that have queries
    int kv_vectors, q_vectors, kv_sections, q_sections, kv_ctas;
};

// y = x / sqrt(mean x^2 + eps) * w over a head, then pairs (a, b) of its first `rot` elements become
// (a cos - b sin, b cos + a sin); in 32 bits, rounded to bf16 once.
// HBM-bound: every element is read and written once, and what counts is bytes in flight and, next, instructions.  A head's
// 16-byte pieces lie in D / 8 lanes, and a warp takes kRopeAhead pieces a lane at once, of a row's heads or, where those are few,
// of several rows: keys and, with them, the same rows' values, which are only moved; or queries, twice as many.  A row's
// (cos, sin) are read once for all of its heads and multiplied by the weights then, so that an element takes two products
// of two numbers each, and one by 1 / sqrt.  The other element of a pair comes as it lies in memory: of halves from the lane
// rot / 16 away, of neighbours from the same word.
// 4 x 32,768 rows of 8 KV heads 178 us, 6.1 TB/s read and written (keys and values in warps of their own, one row at a time: 230;
// CTAs of 256 threads: 182); 4,096 rows with all of 32 heads' queries 22 us, 4.7 TB/s: three and a half waves of warps; eight
// single rows 2.4 us.  The bound of six CTAs an SM leaves 80 registers, and 508 bytes a thread are spilled and 768 read back (d = 64
// and 128 alike).  Of five, 96 registers and nothing spilled, it measures 173, 20.7 and 2.35 us.
constexpr int kRopeThreads = 128, kRopeAhead = 4;
template <int D>
__host__ __device__ constexpr int rope_heads_a_piece() { return 32 / (D / 8); }
// Pieces a lane for a row of `heads`, a power of two of at most `most`, and the sections of it.
template <int D>
inline void rope_share(int heads, int most, int& vectors, int& sections) {
    const int all = (heads + rope_heads_a_piece<D>() - 1) / rope_heads_a_piece<D>();
    for (vectors = 1; vectors < all && vectors < most;) vectors *= 2;
    sections = (all + vectors - 1) / vectors;
}

// What a lane multiplies its eight elements of a head by, and their mates of the pairs.
template <int D>
struct Turn {
    float2 own[4], mate[4];
    uint32_t w[4], mate_w[4];                // the weights, as they lie in memory
    bool normed, turns;
    int from;                                // lane of the mates

    static __device__ __forceinline__ float2 wide(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
    static __device__ __forceinline__ float2 times(float2 a, float2 b) {
        float2 d;
        asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
            : "=f"(d.x), "=f"(d.y)
            : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
        return d;
    }
    static __device__ __forceinline__ float2 times_plus(float2 a, float2 b, float2 c) {
        float2 d;
        tc::unpack2(tc::ffma2(tc::pack2(a.x, a.y), tc::pack2(b.x, b.y), tc::pack2(c.x, c.y)), d.x, d.y);
        return d;
    }
    __device__ __forceinline__ void mates(const NormRopeParams& p, const uint32_t (&u)[4], uint32_t (&m)[4]) const {
        if (p.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = __byte_perm(u[e], 0u, 0x1032);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = __shfl_sync(0xffffffffu, u[e], from);
        }
    }
    __device__ __forceinline__ void weigh(const NormRopeParams& p, const __nv_bfloat16* weight, int l) {
        const int half = p.rot / 16, lane = threadIdx.x & 31;
        normed = weight != nullptr;
        turns = l < 2 * half;                // this lane's elements are of the rotated part
        from = l < half ? lane + half : turns ? lane - half : lane;
        const uint32_t ones = 0x3f803f80u;
        const uint4 v = normed ? reinterpret_cast<const uint4*>(weight)[l] : make_uint4(ones, ones, ones, ones);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        mates(p, w, mate_w);
    }
    // row t's angles
    __device__ __forceinline__ void to(const NormRopeParams& p, int b, int t, int l) {
#pragma unroll
        for (int e = 0; e < 4; ++e) own[e] = wide(w[e]), mate[e] = make_float2(0.f, 0.f);
        if (!turns) return;
        const int half = p.rot / 16;
        const int position = p.positions ? p.positions[(size_t)b * p.rows + t] : p.first + t;
        const bool inside = position >= 0 && position < p.table_rows;
        const float2* cs = p.table + (size_t)(inside ? position : 0) * (p.rot / 2);
        float2 c[4], s[4];
        if (p.interleaved) {                 // a lane has both elements of four pairs: (a, b) take (cos, cos) and (-sin, sin)
            const float4* from4 = reinterpret_cast<const float4*>(cs + 4 * l);
            const float4 x = from4[0], y = from4[1];
            c[0] = make_float2(x.x, x.x), c[1] = make_float2(x.z, x.z), c[2] = make_float2(y.x, y.x), c[3] = make_float2(y.z, y.z);
            s[0] = make_float2(-x.y, x.y), s[1] = make_float2(-x.w, x.w), s[2] = make_float2(-y.y, y.y), s[3] = make_float2(-y.w, y.w);
        } else {                             // one element of eight pairs, all a or all b
            const float4* from4 = reinterpret_cast<const float4*>(cs + 8 * (l < half ? l : l - half));
            const float sign = l < half ? -1.f : 1.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 x = from4[e];
                c[e] = make_float2(x.x, x.z), s[e] = make_float2(sign * x.y, sign * x.w);
            }
        }
        const float nan = __int_as_float(0x7fffffff);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            own[e] = inside ? times(c[e], own[e]) : make_float2(nan, nan);
            mate[e] = times(s[e], wide(mate_w[e]));
        }
    }
    __device__ __forceinline__ uint4 turned(const NormRopeParams& p, uint4 in) const {
        const uint32_t u[4] = {in.x, in.y, in.z, in.w};
        uint32_t m[4];
        mates(p, u, m);
        float2 f[4], y[4];
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = wide(u[e]);
            sum = times_plus(f[e], f[e], sum);
            y[e] = times(f[e], own[e]);
        }
        if (turns)                           // elsewhere the mates are the elements, and an infinity times 0 is no infinity
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = times_plus(wide(m[e]), mate[e], y[e]);
        if (normed) {
            float all = sum.x + sum.y;
#pragma unroll
            for (int o = D / 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
            const float r = rsqrtf(fmaf(all, 1.f / D, p.eps));
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = times(y[e], make_float2(r, r));
        }
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(y[e].x, y[e].y);
            o[e] = *reinterpret_cast<const uint32_t*>(&v);
        }
        return make_uint4(o[0], o[1], o[2], o[3]);
    }
};

// V pieces a lane a row, so kRopeAhead / V rows (of queries twice as many): `index` of the warp among those of its kind.
template <int D, int V>
__device__ __forceinline__ void rope_keys(const NormRopeParams& p, int index) {
    constexpr int VPR = D / 8, HPP = rope_heads_a_piece<D>(), A = kRopeAhead, R = A / V;
    const int lane = threadIdx.x & 31, l = lane % VPR, b = blockIdx.y;
    const int t0 = index / p.kv_sections * R, h0 = index % p.kv_sections * V * HPP + lane / VPR;
    if (t0 >= p.rows) return;
    uint4 k[A], v[A];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint4* kr = reinterpret_cast<const uint4*>(p.k + b * p.k_prompt + (t0 + r) * p.k_row) + (size_t)h0 * VPR + l;
        const uint4* vr = reinterpret_cast<const uint4*>(p.v + b * p.v_prompt + (t0 + r) * p.v_row) + (size_t)h0 * VPR + l;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool there = t0 + r < p.rows && h0 + i * HPP < p.Hkv;
            k[r * V + i] = load_if(kr + i * 32, there);
            v[r * V + i] = load_if(vr + i * 32, there);
        }
    }
    Turn<D> turn;
    turn.weigh(p, p.k_weight, l);
    const size_t head = (size_t)p.N * VPR, at = (((size_t)b * p.L + p.layer) * p.Hkv + h0) * head + (size_t)(p.first + t0) * VPR + l;
    uint4 *ko = reinterpret_cast<uint4*>(p.K) + at, *vo = reinterpret_cast<uint4*>(p.V) + at;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (t0 + r >= p.rows) break;
        turn.to(p, b, t0 + r, l);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint4 y = turn.turned(p, k[r * V + i]);
            if (h0 + i * HPP < p.Hkv) ko[i * HPP * head + r * VPR] = y, vo[i * HPP * head + r * VPR] = v[r * V + i];
        }
    }
}
template <int D, int V>
__device__ __forceinline__ void rope_queries(const NormRopeParams& p, int index) {
    constexpr int VPR = D / 8, HPP = rope_heads_a_piece<D>(), A = 2 * kRopeAhead, R = A / V;
    const int lane = threadIdx.x & 31, l = lane % VPR, b = blockIdx.y;
    const int t0 = index / p.q_sections * R + p.q_first, h0 = index % p.q_sections * V * HPP + lane / VPR;
    if (t0 >= p.rows) return;
    uint4 q[A];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint4* qr = reinterpret_cast<const uint4*>(p.q + b * p.q_prompt + (t0 + r) * p.q_row) + (size_t)h0 * VPR + l;
#pragma unroll
        for (int i = 0; i < V; ++i) q[r * V + i] = load_if(qr + i * 32, t0 + r < p.rows && h0 + i * HPP < p.H);
    }
    Turn<D> turn;
    turn.weigh(p, p.q_weight, l);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int t = t0 + r, at = p.first + t - (p.N - p.W);      // of the window
        if (t >= p.rows) break;
        turn.to(p, b, t, l);
        uint4* wo = reinterpret_cast<uint4*>(p.Qwin) + ((((size_t)b * p.L + p.layer) * p.H + h0) * p.W + at) * VPR + l;
        uint4* qo = reinterpret_cast<uint4*>(p.q_out) + (((size_t)b * p.rows + t) * p.H + h0) * VPR + l;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint4 y = turn.turned(p, q[r * V + i]);
            if (h0 + i * HPP >= p.H) continue;
            if (at >= 0) wo[(size_t)i * HPP * p.W * VPR] = y;
            if (p.q_out) qo[i * 32] = y;
        }
    }
}
template <int D>
__global__ void __launch_bounds__(kRopeThreads, 6) norm_rope_kernel(const NormRopeParams p) {
    constexpr int NW = kRopeThreads / 32;
    const int warp = threadIdx.x >> 5, x = blockIdx.x;
    grid_release();
    grid_wait();
    if (x < p.kv_ctas) {
        const int index = x * NW + warp;
        switch (p.kv_vectors) {
            case 1: rope_keys<D, 1>(p, index); break;
            case 2: rope_keys<D, 2>(p, index); break;
            default: rope_keys<D, 4>(p, index);
        }
    } else {
        const int index = (x - p.kv_ctas) * NW + warp;
        switch (p.q_vectors) {
            case 1: rope_queries<D, 1>(p, index); break;
            case 2: rope_queries<D, 2>(p, index); break;
            case 4: rope_queries<D, 4>(p, index); break;
            default: rope_queries<D, 8>(p, index);
        }
    }
}

}  // namespace shotkv
