// Load-balance loss of the router with per-expert counts, per sequence of a packed batch, and its gradients.
//
//   p[t,e]  = softmax_e(z) or sigmoid(z_e) / sum_e' sigmoid(z_e')          z: logits (+ bias before the score)
//   L_s     = E / (k T_s) sum_e counts[s,e] P[s,e],   P[s,e] = 1 / T_s sum_{t in s} p[t,e]
//   dz[t,e] = p (c_e - sum_e' p c_e') [(1 - s_e) for the sigmoid],   c_e = dloss_s E / (k T_s^2) counts[s,e]
//
// A token is a group of G lanes (four experts a lane, and again G lanes further on where E is above 128), so that a row of the
// logits is read once, in whole vectors, and its maximum and sums are shuffles.  All sums are fp32 in a fixed order: tokens of a
// lane, groups of a warp, warps of a block, blocks of a sequence.  Counts are integers.
#pragma once
#include "common.cuh"
#include "epilogue.cuh"

namespace mop {

// Token ranges of the sequences: off [S+1], non-decreasing (checked nowhere, every use is clamped to [0, T]); null: one, of all tokens.
struct BalSeqs { const int32_t* off; int S, T; };
__device__ __forceinline__ int bal_off(const BalSeqs& q, int i) {
    if (!q.off) return i > 0 ? q.T : 0;
    return min(max(__ldg(q.off + i), 0), q.T);
}
// The sequence of token t: the number of offsets up to t, minus one (-1 before the first sequence, S behind the last).  A warp
// probes 32 places at a time.
__device__ __forceinline__ int bal_find(const BalSeqs& q, int t, int lane) {
    if (!q.off) return 0;
    int lo = 0, hi = q.S + 1;
    while (lo < hi) {
        const int w = (hi - lo + 31) / 32, i = lo + (lane + 1) * w - 1;
        const int n = __popc(__ballot_sync(0xffffffffu, i < hi && bal_off(q, i) <= t));
        const int next = lo + (n + 1) * w - 1;
        lo = min(lo + n * w, hi);
        hi = min(hi, next);
    }
    return lo - 1;
}

struct BalShape { int T, E, k, G, score_fn; bool vec4; };   // G lanes a token; vec4: rows of the logits are whole 16-byte vectors
inline int bal_group(int E) { int g = 2; while (g < 32 && 4 * g < E) g *= 2; return g; }

// Logits of this lane's experts e0 + 4 G v + q; -inf where there is none.
template <int NV>
__device__ __forceinline__ void bal_load(const float* __restrict__ row, const BalShape& s, int e0, bool on, float (&z)[4 * NV]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int e = e0 + 4 * s.G * v;
        if (s.vec4) {
            float4 r = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (on && e < s.E) r = *reinterpret_cast<const float4*>(row + e);
            z[4 * v] = r.x; z[4 * v + 1] = r.y; z[4 * v + 2] = r.z; z[4 * v + 3] = r.w;
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) z[4 * v + q] = on && e + q < s.E ? row[e + q] : -INFINITY;
        }
    }
}
__device__ __forceinline__ float bal_sum(float v, int G) {
    for (int o = G >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// p from z, in place; oms: 1 - sigmoid(z).  A row without a positive score (every expert masked with -inf) has p = 0 throughout.
// Exponentials by ex2 of the scaled argument: 2^-22 relative, and half a step of an argument of at most about 15 more.
template <int NV>
__device__ __forceinline__ void bal_scores(const BalShape& s, float (&z)[4 * NV], float (&oms)[4 * NV]) {
    float sum = 0.0f;
    if (s.score_fn == 0) {
        float m = z[0];
#pragma unroll
        for (int i = 1; i < 4 * NV; ++i) m = fmaxf(m, z[i]);
        for (int o = s.G >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (m == -INFINITY) m = 0.0f;
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) { z[i] = __expf(z[i] - m); sum += z[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            const float e = __expf(-fabsf(z[i])), r = __fdividef(1.0f, 1.0f + e);
            oms[i] = z[i] >= 0.0f ? e * r : r;
            z[i] = z[i] >= 0.0f ? r : (z[i] < 0.0f ? e * r : z[i]);      // (NaN stays)
            sum += z[i];
        }
    }
    sum = bal_sum(sum, s.G);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) z[i] *= inv;
}

// ------------------------------------------------------------------------------------------ forward
// Sequences are cut where blocks of `chunk` tokens end.  A block finishes the sequences that lie inside its chunk; of one that goes
// on beyond it, it leaves the sums: slot 0 where the sequence began before the chunk, slot 1 where it begins in it.
struct BalFwdArgs {
    const float* logits; const float* bias; const int32_t* idx;
    BalSeqs q; BalShape s;
    int chunk;
    int32_t* counts; float* prob; float* loss;
    float* part_p; int32_t* part_c;      // [blocks][2][E]
};
// Sum over the block's threads, in the first one; `sh` holds 32 floats.
__device__ __forceinline__ float bal_block_sum(float v, float* sh) {
    v = bal_sum(v, 32);
    __syncthreads();
    if (threadIdx.x % 32 == 0) sh[threadIdx.x / 32] = v;
    __syncthreads();
    float r = 0.0f;
    if (threadIdx.x == 0)
        for (int w = 0; w < (int)blockDim.x / 32; ++w) r += sh[w];
    return r;
}

template <int NV>
__global__ void __launch_bounds__(512) balance_fwd_kernel(const BalFwdArgs a) {
    pdl_begin();
    extern __shared__ float bal_smem[];                                   // [W][E] sums, [E] counts
    __shared__ float sh[32];
    const BalShape s = a.s;
    const int W = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int tpw = 32 / s.G, in_group = lane % s.G, group = lane / s.G, e0 = 4 * in_group;
    int32_t* cnt = reinterpret_cast<int32_t*>(bal_smem + (size_t)W * s.E);
    for (int e = threadIdx.x; e < s.E; e += blockDim.x) cnt[e] = 0;
    float bias[4 * NV];
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) {
        const int e = e0 + 4 * s.G * (i / 4) + i % 4;
        bias[i] = a.bias && e < s.E ? a.bias[e] : 0.0f;
    }
    const int c0 = blockIdx.x * a.chunk, c1 = min(s.T, c0 + a.chunk);
    const int end = min(c1, bal_off(a.q, a.q.S));
    int t = max(c0, bal_off(a.q, 0));
    __syncthreads();
    while (t < end) {
        const int seq = min(max(bal_find(a.q, t, lane), 0), a.q.S - 1);
        const int first = bal_off(a.q, seq), last = max(bal_off(a.q, seq + 1), t + 1), stop = min(last, end);
        float acc[4 * NV];
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) acc[i] = 0.0f;
        for (int tb = t + warp * tpw; tb < stop; tb += W * tpw) {
            const int mine = tb + group;
            const bool on = mine < stop;
            float z[4 * NV], oms[4 * NV];
            bal_load<NV>(a.logits + (size_t)mine * s.E, s, e0, on, z);
            if (on)
                for (int j = in_group; j < s.k; j += s.G) {
                    const int e = a.idx[(size_t)mine * s.k + j];
                    if (e >= 0 && e < s.E) atomicAdd(&cnt[e], 1);         // integers: any order gives the same counts
                }
            if (a.bias)
#pragma unroll
                for (int i = 0; i < 4 * NV; ++i) z[i] += bias[i];
            bal_scores<NV>(s, z, oms);
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) acc[i] += on ? z[i] : 0.0f;
        }
        for (int o = s.G; o < 32; o <<= 1)
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
        if (group == 0)
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) {
                const int e = e0 + 4 * s.G * (i / 4) + i % 4;
                if (e < s.E) bal_smem[(size_t)warp * s.E + e] = acc[i];
            }
        __syncthreads();
        const bool whole = first >= c0 && last <= c1;
        const float n = (float)max(1, last - first);
        const size_t slot = ((size_t)blockIdx.x * 2 + (first < c0 ? 0 : 1)) * s.E;
        float dot = 0.0f;
        for (int e = threadIdx.x; e < s.E; e += blockDim.x) {
            float p = 0.0f;
            for (int w = 0; w < W; ++w) p += bal_smem[(size_t)w * s.E + e];
            const int32_t c = cnt[e];
            cnt[e] = 0;
            if (whole) {
                p /= n;
                a.prob[(size_t)seq * s.E + e] = p;
                a.counts[(size_t)seq * s.E + e] = c;
                dot = fmaf((float)c, p, dot);
            } else {
                a.part_p[slot + e] = p;
                a.part_c[slot + e] = c;
            }
        }
        if (whole) {
            dot = bal_block_sum(dot, sh);
            if (threadIdx.x == 0) a.loss[seq] = dot * ((float)s.E / ((float)s.k * n));
        }
        __syncthreads();
        t = stop;
    }
}

// The sequences that several blocks hold a part of, and those without tokens.  Thread (slice, e) adds every slices-th block's sums.
__global__ void __launch_bounds__(1024) balance_finish_kernel(const BalFwdArgs a) {
    pdl_begin();
    __shared__ float sh[32];
    __shared__ float sp[1024];
    __shared__ int32_t sc[1024];
    const int E = a.s.E, Ep = (E + 31) / 32 * 32, slices = (int)blockDim.x / Ep;
    const int e = threadIdx.x % Ep, slice = threadIdx.x / Ep;
    for (int seq = blockIdx.x; seq < a.q.S; seq += gridDim.x) {
        const int first = bal_off(a.q, seq), last = bal_off(a.q, seq + 1);
        const int b0 = first / a.chunk, b1 = (last - 1) / a.chunk;
        if (last > first && b0 == b1) continue;                           // done by its block
        float p = 0.0f;
        int32_t c = 0;
        if (last > first && slice < slices && e < E)
#pragma unroll 8
            for (int b = b0 + slice; b <= b1; b += slices) {
                const size_t slot = ((size_t)b * 2 + (b == b0 ? 1 : 0)) * E + e;
                p += a.part_p[slot];
                c += a.part_c[slot];
            }
        sp[threadIdx.x] = p;
        sc[threadIdx.x] = c;
        __syncthreads();
        float dot = 0.0f;
        const float n = (float)max(1, last - first);
        if (slice == 0 && e < E) {
            for (int i = 1; i < slices; ++i) { p += sp[i * Ep + e]; c += sc[i * Ep + e]; }
            p /= n;
            a.prob[(size_t)seq * E + e] = p;
            a.counts[(size_t)seq * E + e] = c;
            dot = (float)c * p;
        }
        dot = bal_block_sum(dot, sh);
        if (threadIdx.x == 0) a.loss[seq] = dot * ((float)E / ((float)a.s.k * n));
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------ backward
struct BalBwdArgs {
    const float* logits; const float* bias; const int32_t* counts; const float* dloss;
    BalSeqs q; BalShape s;
    int chunk;
    float* dz;                            // [T, E]: the caller's dlogits, or the workspace
    float* dbias_part;                    // [blocks][E] or null
};
// dz, zero for tokens outside the sequences.  Counts are taken relative to their mean (k T_s / E, rounded): c_e - sum p c does not
// change by a shift, and under a nearly balanced load, which this loss aims at, the difference keeps its digits.
template <int NV>
__global__ void __launch_bounds__(NV == 8 ? 256 : 512) balance_dz_kernel(const BalBwdArgs a) {
    pdl_begin();
    extern __shared__ float bal_smem[];                                   // [W][E]
    const BalShape s = a.s;
    const int W = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int tpw = 32 / s.G, in_group = lane % s.G, group = lane / s.G, e0 = 4 * in_group;
    const int c0 = blockIdx.x * a.chunk, c1 = min(s.T, c0 + a.chunk);
    float bias[4 * NV], acc[4 * NV];
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) {
        const int e = e0 + 4 * s.G * (i / 4) + i % 4;
        bias[i] = a.bias && e < s.E ? a.bias[e] : 0.0f;
        acc[i] = 0.0f;
    }
    for (int tb = c0 + warp * tpw; tb < c1; tb += W * tpw) {
        const int t = tb + group;
        int seq = bal_find(a.q, tb, lane);
        while (seq < a.q.S && t >= bal_off(a.q, seq + 1)) ++seq;
        const bool on = t < c1 && seq >= 0 && seq < a.q.S;
        float z[4 * NV], oms[4 * NV], c[4 * NV];
        bal_load<NV>(a.logits + (size_t)t * s.E, s, e0, on, z);
        float w = 0.0f, dot = 0.0f;
        int32_t shift = 0;
        if (on) {
            const float n = (float)max(1, bal_off(a.q, seq + 1) - bal_off(a.q, seq));
            w = a.dloss[seq] * ((float)s.E / (float)s.k) / (n * n);
            shift = (int32_t)rintf(n * (float)s.k / (float)s.E);
        }
        if (a.bias)
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) z[i] += bias[i];
        bal_scores<NV>(s, z, oms);
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            const int e = e0 + 4 * s.G * (i / 4) + i % 4;
            c[i] = on && e < s.E ? (float)(a.counts[(size_t)seq * s.E + e] - shift) : 0.0f;
            dot = fmaf(z[i], c[i], dot);
        }
        dot = bal_sum(dot, s.G);
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            const int e = e0 + 4 * s.G * (i / 4) + i % 4;
            float v = w * z[i] * (c[i] - dot);
            if (s.score_fn != 0) v *= oms[i];
            if (!on) v = 0.0f;
            if (t < c1 && e < s.E) a.dz[(size_t)t * s.E + e] = v;
            acc[i] += e < s.E && t < c1 ? v : 0.0f;
        }
    }
    if (!a.dbias_part) return;
    for (int o = s.G; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], o);
    if (group == 0)
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            const int e = e0 + 4 * s.G * (i / 4) + i % 4;
            if (e < s.E) bal_smem[(size_t)warp * s.E + e] = acc[i];
        }
    __syncthreads();
    for (int e = threadIdx.x; e < s.E; e += blockDim.x) {
        float v = 0.0f;
        for (int i = 0; i < W; ++i) v += bal_smem[(size_t)i * s.E + e];
        a.dbias_part[(size_t)blockIdx.x * s.E + e] = v;
    }
}
__global__ void __launch_bounds__(256) balance_dbias_kernel(const float* __restrict__ part, float* __restrict__ dbias, int blocks, int E,
                                                            int accumulate) {
    pdl_begin();
    const int e = blockIdx.x * blockDim.x + threadIdx.x;
    if (e >= E) return;
    float v = 0.0f;
    for (int b = 0; b < blocks; ++b) v += part[(size_t)b * E + e];
    dbias[e] = accumulate ? dbias[e] + v : v;
}

// dW_r = x^T dz over the tokens of the sequences; 64 x 64 outputs a block, 4 x 4 a thread.
__global__ void __launch_bounds__(256) balance_dw_kernel(const bf16* __restrict__ x, const float* __restrict__ dz, const BalSeqs q,
                                                         float* __restrict__ dW, int d, int E, int accumulate) {
    pdl_begin();
    __shared__ float sx[16][64], sz[16][64];
    const int i0 = blockIdx.x * 64, e0 = blockIdx.y * 64, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int begin = bal_off(q, 0), end = bal_off(q, q.S);
    float acc[4][4] = {};
    for (int t0 = begin; t0 < end; t0 += 16) {
        for (int j = threadIdx.x; j < 16 * 64; j += 256) {
            const int t = t0 + j / 64, c = j % 64;
            sx[j / 64][c] = t < end && i0 + c < d ? __bfloat162float(x[(size_t)t * d + i0 + c]) : 0.0f;
            sz[j / 64][c] = t < end && e0 + c < E ? dz[(size_t)t * E + e0 + c] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sx[r][ty * 4 + a], sz[r][tx * 4 + b], acc[a][b]);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int i = i0 + ty * 4 + a, e = e0 + tx * 4 + b;
            if (i < d && e < E) {
                float* o = dW + (size_t)i * E + e;
                *o = accumulate ? *o + acc[a][b] : acc[a][b];
            }
        }
}
// dX (+)= dz W_r^T, rounded to bf16 once.  Rows outside the sequences: zero, or left as they are.
__global__ void __launch_bounds__(256) balance_dx_kernel(const float* __restrict__ dz, const float* __restrict__ W_r, const BalSeqs q,
                                                         bf16* __restrict__ dX, int T, int d, int E, int accumulate) {
    pdl_begin();
    __shared__ float sz[64][17], sw[64][17];
    const int i0 = blockIdx.x * 64, t0 = blockIdx.y * 64, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int begin = bal_off(q, 0), end = bal_off(q, q.S);
    float acc[4][4] = {};
    for (int e0 = 0; e0 < E; e0 += 16) {
        for (int j = threadIdx.x; j < 16 * 64; j += 256) {
            const int r = j / 16, c = j % 16;
            sz[r][c] = t0 + r < T && e0 + c < E ? dz[(size_t)(t0 + r) * E + e0 + c] : 0.0f;
            sw[r][c] = i0 + r < d && e0 + c < E ? W_r[(size_t)(i0 + r) * E + e0 + c] : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 16; ++c)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sz[ty * 4 + a][c], sw[tx * 4 + b][c], acc[a][b]);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int t = t0 + ty * 4 + a, i = i0 + tx * 4 + b;
            if (t >= T || i >= d) continue;
            bf16* o = dX + (size_t)t * d + i;
            const bool inside = t >= begin && t < end;
            if (!accumulate) *o = __float2bfloat16_rn(inside ? acc[a][b] : 0.0f);
            else if (inside) *o = __float2bfloat16_rn(__bfloat162float(*o) + acc[a][b]);
        }
}

// ------------------------------------------------------------------------------------------ host
// Tokens per block: one block for each SM, at least 16 tokens each.
inline int bal_chunk(int T) { const int c = (T + 147) / 148; return c < 16 ? 16 : c; }
inline int bal_blocks(int T) { return (T + bal_chunk(T) - 1) / bal_chunk(T); }
inline int bal_warps(int E) { return E <= 512 ? 16 : 8; }
inline size_t bal_smem_bytes(int E, int warps) { return (size_t)(warps + 1) * E * 4; }
inline BalShape bal_shape(const mop_moe_shape& s) {
    return {s.T, s.E, s.k, bal_group(s.E), s.score_fn, s.E % 4 == 0};
}
#define BAL_BY_WIDTH(E, GO)                                       \
    do {                                                          \
        if ((E) <= 128) GO(1);                                    \
        else if ((E) <= 256) GO(2);                               \
        else if ((E) <= 512) GO(4);                               \
        else GO(8);                                               \
    } while (0)

}  // namespace mop
