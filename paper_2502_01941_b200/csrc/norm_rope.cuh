// From a layer's projection to the tensors that the other calls take: queries and keys normed per head and rotated by
// position, values as they are, each written in its place.
#pragma once
#include "common.cuh"

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
    int kv_items, items;                     // warps' work: keys and values first, then queries
    int q_sections, kv_sections;             // sections of heads
};

// y = x / sqrt(mean x^2 + eps) * w over a head, then pairs (a, b) of its first `rot` elements become
// (a cos - b sin, b cos + a sin); in 32 bits, rounded to bf16 once.
// HBM-bound: every element is read and written once.  A head's 16-byte pieces lie in D / 8 lanes, and a warp takes
// kAhead * 32 * 8 / D heads of one token, kAhead loads a lane in flight; their (cos, sin) are read once for all of
// them.  Halves as pairs: the other element lies in a lane rot / 16 away, at the same place.
constexpr int kRopeThreads = 256, kRopeAhead = 4;
template <int D>
__global__ void __launch_bounds__(kRopeThreads) norm_rope_kernel(const NormRopeParams p) {
    constexpr int VPR = D / 8, HPW = 32 / VPR, SECTION = kRopeAhead * HPW;
    const int lane = threadIdx.x & 31, l = lane % VPR, sub = lane / VPR;
    int item = blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
    grid_release();
    grid_wait();
    if (item >= p.items) return;
    // what this warp takes: 0 keys, 1 values, 2 queries; of which token; which heads
    int what, b, t, section;
    if (item < p.kv_items) {
        section = item % p.kv_sections;
        item /= p.kv_sections;
        what = item & 1;
        item >>= 1;
        b = item / p.rows;
        t = item - b * p.rows;
    } else {
        item -= p.kv_items;
        what = 2;
        section = item % p.q_sections;
        item /= p.q_sections;
        b = item / (p.rows - p.q_first);
        t = item - b * (p.rows - p.q_first) + p.q_first;
    }
    const int heads = what == 2 ? p.H : p.Hkv;
    const __nv_bfloat16* x = what == 2 ? p.q + b * p.q_prompt + t * p.q_row
                             : what == 1 ? p.v + b * p.v_prompt + t * p.v_row : p.k + b * p.k_prompt + t * p.k_row;
    const uint4* row = reinterpret_cast<const uint4*>(x) + l;
    uint4 in[kRopeAhead];
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i) {
        const int h = section * SECTION + i * HPW + sub;
        in[i] = load_if(row + (size_t)h * VPR, h < heads);
    }
    const int at = p.first + t;              // the token's place in the prompt
    if (what == 1) {
#pragma unroll
        for (int i = 0; i < kRopeAhead; ++i) {
            const int h = section * SECTION + i * HPW + sub;
            if (h < heads) reinterpret_cast<uint4*>(p.V)[((((size_t)b * p.L + p.layer) * p.Hkv + h) * p.N + at) * VPR + l] = in[i];
        }
        return;
    }
    // this lane's eight (cos, sin): of halves those of its elements, of neighbours the first four
    float c[8] = {}, s[8] = {};
    const int half = p.rot / 16;             // lanes of half the rotated part
    if (l < 2 * half) {
        const int position = p.positions ? p.positions[(size_t)b * p.rows + t] : at;
        if (position < 0 || position >= p.table_rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = s[e] = __int_as_float(0x7fffffff);
        } else {
            const float2* cs = p.table + (size_t)position * (p.rot / 2);
            const float4* from = reinterpret_cast<const float4*>(cs + (p.interleaved ? 4 * l : 8 * (l < half ? l : l - half)));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (p.interleaved && e >= 2) break;
                const float4 w = from[e];
                c[2 * e] = w.x, s[2 * e] = w.y, c[2 * e + 1] = w.z, s[2 * e + 1] = w.w;
            }
        }
    }
    const __nv_bfloat16* weight = what == 2 ? p.q_weight : p.k_weight;
    float w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.f;
    const auto widen = [](uint4 v, float (&f)[8]) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) f[2 * e] = __uint_as_float(u[e] << 16), f[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    };
    if (weight) widen(reinterpret_cast<const uint4*>(weight)[l], w);
    const int mate = l < half ? lane + half : l < 2 * half ? lane - half : lane;
#pragma unroll
    for (int i = 0; i < kRopeAhead; ++i) {
        const int h = section * SECTION + i * HPW + sub;
        float f[8], y[8];
        widen(in[i], f);
        if (weight) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(f[e], f[e], sum);
#pragma unroll
            for (int o = VPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float r = rsqrtf(fmaf(sum, 1.f / D, p.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= r * w[e];
        }
        if (p.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[2 * e] = f[2 * e] * c[e] - f[2 * e + 1] * s[e];
                y[2 * e + 1] = f[2 * e + 1] * c[e] + f[2 * e] * s[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float other = __shfl_sync(0xffffffffu, f[e], mate);
                y[e] = f[e] * c[e] + (l < half ? -other : other) * s[e];
            }
        }
        if (l >= 2 * half)                   // past the rotated part (an infinity times a sine of 0 is no infinity)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = f[e];
        if (h >= heads) continue;
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(y[2 * e], y[2 * e + 1]);
            u[e] = *reinterpret_cast<const uint32_t*>(&v);
        }
        const uint4 out = make_uint4(u[0], u[1], u[2], u[3]);
        if (what == 0) {
            reinterpret_cast<uint4*>(p.K)[((((size_t)b * p.L + p.layer) * p.Hkv + h) * p.N + at) * VPR + l] = out;
        } else {
            if (at >= p.N - p.W) reinterpret_cast<uint4*>(p.Qwin)[((((size_t)b * p.L + p.layer) * p.H + h) * p.W + at - (p.N - p.W)) * VPR + l] = out;
            if (p.q_out) reinterpret_cast<uint4*>(p.q_out)[(((size_t)b * p.rows + t) * p.H + h) * VPR + l] = out;
        }
    }
}

}  // namespace shotkv
