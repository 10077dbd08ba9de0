// Load-balance loss of the router with per-expert counts, per sequence of a packed batch, and its gradients.
//
//   p[t,e]  = softmax_e(z) or sigmoid(z_e) / sum_e' sigmoid(z_e')          z: logits (+ bias before the score)
//   L_s     = E / (k T_s) sum_e counts[s,e] P[s,e],   P[s,e] = 1 / T_s sum_{t in s} p[t,e]
//   dz[t,e] = p (c_e - sum_e' p c_e') [(1 - s_e) for the sigmoid],   c_e = dloss_s E / (k T_s^2) counts[s,e]
//
// A token is a group of G lanes (four experts a lane, and again G lanes further on where E is above 128), so that a row of the
// logits is read once, in whole vectors, and its maximum and sums are shuffles.  All sums are fp32 in a fixed order: tokens of a
// lane, groups of a warp, warps of a block, blocks of a sequence.  Counts are integers.
//
// The two products of the backward have T d E multiply-adds each (60 GFLOP at T = 16384, d = 7168, E = 256) and run on the tensor cores:
//   dW_r = x^T dz   must have fp32 accuracy: dz goes in as three bf16 pieces (24 bits), x is bf16 already (bal_dw_pair_kernel)
//   dX = dz W_r^T   is rounded to bf16: both operands go in as fp16 (11 bits), a token's row and 32 rows of W_r scaled by a power of two, so that
//                   neither the size of the upstream weight nor that of the router's weights matters (vd_gemm_kernel, kind VD_R)
#pragma once
#include <cuda_fp16.h>

#include "distill.cuh"

namespace mop {

// Token ranges of the sequences: off [S+1], non-decreasing (checked nowhere, every use is clamped to [0, T]); null: one, of all tokens.
struct BalSeqs { const int32_t* off; int S, T; };
__device__ __forceinline__ int bal_off(const BalSeqs& q, int i) {
    if (!q.off) return i > 0 ? q.T : 0;
    return min(max(q.off[i], 0), q.T);
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
__device__ __forceinline__ void bal_load(const float* row, const BalShape& s, int e0, bool on, float (&z)[4 * NV]) {
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
        // The scores of a row that lies far below zero are taken relative to its largest: below -87 they, and below -88 the reciprocal of
        // their sum, leave the range of fp32.  (Such a row: no lane of the group has a logit of -16 or more.)
        float m = z[0], shift = 0.0f;
#pragma unroll
        for (int i = 1; i < 4 * NV; ++i) m = fmaxf(m, z[i]);
        const uint32_t near = __ballot_sync(0xffffffffu, m >= -16.0f);
        const bool far = (near & (0xffffffffu >> (32 - s.G)) << (threadIdx.x % 32 & ~(s.G - 1))) == 0;
        if (__any_sync(0xffffffffu, far)) {
            for (int o = s.G >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            if (far && m > -INFINITY) shift = m;
        }
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            const float e = __expf(-fabsf(z[i])), r = __fdividef(1.0f, 1.0f + e);
            oms[i] = z[i] >= 0.0f ? e * r : r;
            z[i] = z[i] >= 0.0f ? r : (z[i] < 0.0f ? (shift == 0.0f ? e : __expf(z[i] - shift)) * r : z[i]);      // (NaN stays)
            sum += z[i];
        }
    }
    sum = bal_sum(sum, s.G);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) z[i] *= inv;
}

// ------------------------------------------------------------------------------------------ forward
// Bound by latency: T 16384, E 256 takes 12 us for 17.8 MB (a launch, the search for the block's sequence, three or four rounds of one
// row per warp, 16 warps' sums through shared memory), T 256, E 8 in one block 5.8.  In a training loop the calls themselves take
// 16 us with one launch and 19 with two, about what the two kernels of the former, one after the other, take as well (12 + 7.6).
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
        // a row of logits, and the lane's pick, are fetched one round ahead
        float next[4 * NV];
        int pick = -1;
        auto fetch = [&](int tb) {
            const int mine = tb + group;
            const bool on = mine < stop;
            bal_load<NV>(a.logits + (size_t)mine * s.E, s, e0, on, next);
            pick = on && in_group < s.k ? a.idx[(size_t)mine * s.k + in_group] : -1;
        };
        fetch(t + warp * tpw);
        for (int tb = t + warp * tpw; tb < stop; tb += W * tpw) {
            const int mine = tb + group, e_pick = pick;
            const bool on = mine < stop;
            float z[4 * NV], oms[4 * NV];
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) z[i] = next[i];
            fetch(tb + W * tpw);
            if (e_pick >= 0 && e_pick < s.E) atomicAdd(&cnt[e_pick], 1);   // integers: any order gives the same counts
            if (on)
                for (int j = in_group + s.G; j < s.k; j += s.G) {
                    const int e = a.idx[(size_t)mine * s.k + j];
                    if (e >= 0 && e < s.E) atomicAdd(&cnt[e], 1);
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
    if (gridDim.x > 1) return;
    // a single block: no other kernel follows, so the sequences without tokens are its own
    for (int seq = warp; seq < a.q.S; seq += W) {
        if (bal_off(a.q, seq + 1) > bal_off(a.q, seq)) continue;
        for (int e = lane; e < s.E; e += 32) { a.prob[(size_t)seq * s.E + e] = 0.0f; a.counts[(size_t)seq * s.E + e] = 0; }
        if (lane == 0) a.loss[seq] = 0.0f;
    }
}

// The sequences that several blocks hold a part of, and those without tokens: a cluster each, whose CTAs share the experts (the
// partial sums of a long batch are 600 KB at 256 experts, 5 us for one SM alone: 11.3 us in one CTA, 7.6 in eight).  Thread (slice, vector) adds every
// slices-th block's sums of four experts (of one where the rows are no whole vectors); the CTAs' shares of the loss meet in the first
// one's shared memory.
constexpr int BF_THREADS = 512, BF_CLUSTER = 8;
__global__ void __launch_bounds__(BF_THREADS) balance_finish_kernel(const BalFwdArgs a) {
    cluster_sync_all();          // the first CTA has started before anything is written to its shared memory
    pdl_begin();
    __shared__ float sh[32], share[BF_CLUSTER];
    __shared__ __align__(16) float sp[4 * BF_THREADS];
    __shared__ __align__(16) int32_t sc[4 * BF_THREADS];
    uint32_t ctas;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ctas));
    const uint32_t rank = cluster_ctarank();
    const int E = a.s.E, per = a.s.vec4 ? 4 : 1, all = E / per, mine = (all + (int)ctas - 1) / (int)ctas;
    const int v0 = min(all, (int)rank * mine), vecs = max(1, min(all, v0 + mine) - v0);      // (a CTA without any repeats one, unused)
    const int e0 = v0 * per, ne = (min(all, v0 + mine) - v0) * per;
    const int slices = BF_THREADS / vecs, vec = threadIdx.x % vecs, slice = threadIdx.x / vecs, tid = threadIdx.x, row = vecs * per;
    for (int seq = blockIdx.x / ctas; seq < a.q.S; seq += gridDim.x / ctas) {
        const int first = bal_off(a.q, seq), last = bal_off(a.q, seq + 1);
        const int b0 = first / a.chunk, b1 = (last - 1) / a.chunk;
        if (last > first && b0 == b1) continue;                           // done by its block (for every CTA of the cluster alike)
        float dot = 0.0f;
        const float n = (float)max(1, last - first);
        {
            float4 p = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            int4 c = make_int4(0, 0, 0, 0);
            if (last > first && slice < slices && ne > 0) {
                if (per == 4) {
#pragma unroll 6
                    for (int b = b0 + slice; b <= b1; b += slices) {
                        const size_t slot = ((size_t)b * 2 + (b == b0 ? 1 : 0)) * E + e0 + 4 * vec;
                        const float4 x = *reinterpret_cast<const float4*>(a.part_p + slot);
                        const int4 y = *reinterpret_cast<const int4*>(a.part_c + slot);
                        p.x += x.x; p.y += x.y; p.z += x.z; p.w += x.w;
                        c.x += y.x; c.y += y.y; c.z += y.z; c.w += y.w;
                    }
                } else {
#pragma unroll 8
                    for (int b = b0 + slice; b <= b1; b += slices) {
                        const size_t slot = ((size_t)b * 2 + (b == b0 ? 1 : 0)) * E + e0 + vec;
                        p.x += a.part_p[slot];
                        c.x += a.part_c[slot];
                    }
                }
            }
            if (slice < slices) {
                if (per == 4) {
                    *reinterpret_cast<float4*>(sp + 4 * tid) = p;
                    *reinterpret_cast<int4*>(sc + 4 * tid) = c;
                } else { sp[tid] = p.x; sc[tid] = c.x; }
            }
            __syncthreads();
            for (int e = tid; e < ne; e += BF_THREADS) {                  // slice i holds its sums `row` further on
                float q = 0.0f;
                int32_t d = 0;
                for (int i = 0; i < slices; ++i) { q += sp[i * row + e]; d += sc[i * row + e]; }
                q /= n;
                a.prob[(size_t)seq * E + e0 + e] = q;
                a.counts[(size_t)seq * E + e0 + e] = d;
                dot = fmaf((float)d, q, dot);
            }
        }
        dot = bal_block_sum(dot, sh);
        if (tid == 0) {
            uint32_t to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(share + rank)));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(dot) : "memory");
        }
        __syncwarp();
        cluster_sync_all();
        if (tid == 0 && rank == 0) {
            float total = 0.0f;
            for (uint32_t i = 0; i < ctas; ++i) total += share[i];
            a.loss[seq] = total * ((float)E / ((float)a.s.k * n));
        }
        __syncwarp();
        cluster_sync_all();                       // (also: nobody leaves while another may still write to it)
    }
}

// ------------------------------------------------------------------------------------------ backward
struct BalBwdArgs {
    const float* logits; const float* bias; const int32_t* counts; const float* dloss;
    BalSeqs q; BalShape s;
    int chunk, dz_blocks;
    int32_t* note;                        // cleared here: the word of the PdlNote between the two products
    float* dz;                            // [T, E] fp32, or null
    float* dbias_part;                    // [dz_blocks][E], or null
    // for the tensor cores, each or null:
    int Ep;                               // columns of the buffers below: E rounded up to 64, zeros behind it
    bf16* pieces;                         // [3][T][Ep]: dz = hi + mid + lo
    __half* dz16; float* row_scale;       // [T][Ep], [T]: dz = dz16 row_scale
    const float* W_r; __half* w16; float* col_scale; int d;      // [d][Ep], [d / 32]: W_r = w16 col_scale, by the blocks behind dz_blocks
    const uint4* x; uint4* xe;            // [128][d]: the first and last 64 tokens of the sequences' range, see bal_dw_pair_kernel
};
constexpr int BAL_EDGE_BLOCKS = 8;        // blocks for each of the two edges of x
inline __host__ __device__ int bal_ep(int E) { return (E + 63) / 64 * 64; }

// The power of two that brings a row's largest magnitude into [2^14, 2^15), and its reciprocal; fp16 then keeps 11 bits of what is
// within 2^-28 of that, and the products' fp32 sums cannot overflow.
__device__ __forceinline__ void bal_scale(float amax, float& up, float& down) {
    const int e = (int)((__float_as_uint(amax) >> 23) & 255u) - 127;
    const int by = min(14 - e, 126);
    up = __uint_as_float((uint32_t)(by + 127) << 23);
    down = __uint_as_float((uint32_t)(127 - by) << 23);
}
__device__ __forceinline__ uint2 bal_half4(const float* v, float by) {
    const __half2 a = __floats2half2_rn(v[0] * by, v[1] * by), b = __floats2half2_rn(v[2] * by, v[3] * by);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
// 32 rows of W_r a block: fp16 with one scale for all of them (a row that is 2^-28 of its neighbours would lose digits).
__device__ __forceinline__ void bal_convert_w(const BalBwdArgs& a, int block, int blocks) {
    __shared__ float amax_of[16];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32, E = a.s.E;
    for (int r0 = block * 32; r0 < a.d; r0 += blocks * 32) {
        float amax = 0.0f, up, down;
        for (int r = r0 + warp; r < min(r0 + 32, a.d); r += warps)
#pragma unroll 4
            for (int e = lane; e < E; e += 32) {
                const float w = fabsf(a.W_r[(size_t)r * E + e]);
                amax = fmaxf(amax, w < INFINITY ? w : 0.0f);       // (an infinity stays one, the rows beside it keep their digits)
            }
        for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        __syncthreads();
        if (lane == 0) amax_of[warp] = amax;
        __syncthreads();
        for (int w = 0; w < warps; ++w) amax = fmaxf(amax, amax_of[w]);
        bal_scale(amax, up, down);
        for (int r = r0 + warp; r < min(r0 + 32, a.d); r += warps)
            for (int e = 4 * lane; e < a.Ep; e += 128) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = e + i < E ? a.W_r[(size_t)r * E + e + i] : 0.0f;
                *reinterpret_cast<uint2*>(a.w16 + (size_t)r * a.Ep + e) = bal_half4(v, up);
            }
        if (threadIdx.x == 0) a.col_scale[r0 / 32] = down;
    }
}
// Blocks of 64 tokens that the range [begin, end) of the sequences covers in part only: the padding in them must not meet the
// products (0 x NaN), so such a block is copied, with zeros in the padding's place, and read from the copy.
__device__ __forceinline__ bool bal_dirty(int kb, int begin, int end, int T) { return kb * 64 < begin || min(kb * 64 + 64, T) > end; }
__device__ __forceinline__ void bal_copy_edge(const BalBwdArgs& a, int edge, int block) {
    const int begin = bal_off(a.q, 0), end = bal_off(a.q, a.q.S);
    if (begin >= end) return;
    const int first = begin / 64, kb = edge ? (end - 1) / 64 : first;
    if ((edge && kb == first) || !bal_dirty(kb, begin, end, a.s.T)) return;
    const int per = a.d / 8;
    for (int i = block * blockDim.x + threadIdx.x; i < 64 * per; i += BAL_EDGE_BLOCKS * blockDim.x) {
        const int t = kb * 64 + i / per;
        a.xe[(size_t)edge * 64 * per + i] = t >= begin && t < end ? a.x[(size_t)t * per + i % per] : make_uint4(0, 0, 0, 0);
    }
}

// T 16384, d 7168, E 256: 24 us for 17 MB in and 41 MB out, beside it 7.3 MB of W_r; rounds of about a microsecond, three blocks of eight
// warps on an SM.
// dz, zero for tokens outside the sequences.  Counts are taken relative to their mean (k T_s / E, rounded): c_e - sum p c does not
// change by a shift, and under a nearly balanced load, which this loss aims at, the difference keeps its digits.
// The blocks behind the first dz_blocks prepare W_r and the edges of x.
template <int NV, bool PRE>
__global__ void __launch_bounds__(256, NV <= 2 ? 3 : NV == 4 ? 2 : 1) balance_dz_kernel(const BalBwdArgs a) {
    pdl_begin();
    extern __shared__ float bal_smem[];                                   // [W][E]
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.note = 0;
    if ((int)blockIdx.x >= a.dz_blocks) {
        int b = (int)blockIdx.x - a.dz_blocks;
        if (a.xe) {
            if (b < 2 * BAL_EDGE_BLOCKS) { bal_copy_edge(a, b / BAL_EDGE_BLOCKS, b % BAL_EDGE_BLOCKS); return; }
            b -= 2 * BAL_EDGE_BLOCKS;
        }
        bal_convert_w(a, b, (int)gridDim.x - a.dz_blocks - (a.xe ? 2 * BAL_EDGE_BLOCKS : 0));
        return;
    }
    const BalShape s = a.s;
    const int W = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int tpw = 32 / s.G, in_group = lane % s.G, group = lane / s.G, e0 = 4 * in_group;
    const int c0 = blockIdx.x * a.chunk, c1 = min(s.T, c0 + a.chunk);
    float bias[PRE ? 4 * NV : 1], acc[PRE ? 4 * NV : 1];
    if constexpr (PRE)
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            const int e = e0 + 4 * s.G * (i / 4) + i % 4;
            bias[i] = e < s.E ? a.bias[e] : 0.0f;
            acc[i] = 0.0f;
        }
    // the lane's sequence, and what follows from it, as long as its tokens stay inside
    int first = 0, last = 0;
    float w = 0.0f, c[4 * NV], next[4 * NV];
    bal_load<NV>(a.logits + (size_t)(c0 + warp * tpw + group) * s.E, s, e0, c0 + warp * tpw + group < c1, next);
    for (int tb = c0 + warp * tpw; tb < c1; tb += W * tpw) {
        const int t = tb + group;
        float z[4 * NV], oms[4 * NV], dot = 0.0f;
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) z[i] = next[i];
        bal_load<NV>(a.logits + (size_t)(t + W * tpw) * s.E, s, e0, t + W * tpw < c1, next);
        if (__any_sync(0xffffffffu, t < c1 && !(t >= first && t < last))) {
            int seq = bal_find(a.q, tb, lane);
            while (seq < a.q.S && t >= bal_off(a.q, seq + 1)) ++seq;
            const bool in = t < c1 && seq >= 0 && seq < a.q.S;
            first = last = 0;
            int32_t shift = 0;
            if (in) {
                first = bal_off(a.q, seq); last = bal_off(a.q, seq + 1);
                const float n = (float)max(1, last - first);
                w = a.dloss[seq] * ((float)s.E / (float)s.k) / (n * n);
                shift = (int32_t)rintf(n * (float)s.k / (float)s.E);
            }
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) {
                const int e = e0 + 4 * s.G * (i / 4) + i % 4;
                c[i] = in && e < s.E ? (float)(a.counts[(size_t)seq * s.E + e] - shift) : 0.0f;
            }
        }
        const bool on = t >= first && t < last && t < c1;
        if (!on)
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) z[i] = -INFINITY;            // (a padding token's logits may be anything)
        if constexpr (PRE)
#pragma unroll
            for (int i = 0; i < 4 * NV; ++i) z[i] += bias[i];
        bal_scores<NV>(s, z, oms);
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) dot = fmaf(z[i], c[i], dot);
        dot = bal_sum(dot, s.G);
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
            float v = w * z[i] * (c[i] - dot);
            if (s.score_fn != 0) v *= oms[i];
            const bool there = on && e0 + 4 * s.G * (i / 4) + i % 4 < s.E;
            z[i] = there ? v : 0.0f;
            if constexpr (PRE) acc[i] += z[i];
            amax = fmaxf(amax, fabsf(z[i]));
        }
        if (a.dz && t < c1)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = e0 + 4 * s.G * v;
                float* o = a.dz + (size_t)t * s.E + e;
                if (s.vec4) {
                    if (e < s.E) *reinterpret_cast<float4*>(o) = make_float4(z[4 * v], z[4 * v + 1], z[4 * v + 2], z[4 * v + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (e + i < s.E) o[i] = z[4 * v + i];
                }
            }
        if (a.dz16) {
            float up, down;
            for (int o = s.G >> 1; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            bal_scale(amax, up, down);
            if (t < c1) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const int e = e0 + 4 * s.G * v;
                    if (e < a.Ep) *reinterpret_cast<uint2*>(a.dz16 + (size_t)t * a.Ep + e) = bal_half4(z + 4 * v, up);
                }
                if (in_group == 0) a.row_scale[t] = down;
            }
        }
        if (a.pieces && t < c1)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int e = e0 + 4 * s.G * v;
                if (e >= a.Ep) continue;
#pragma unroll
                for (int piece = 0; piece < 3; ++piece) {
                    const uint2 r = make_uint2(pack_bf16x2(z[4 * v], z[4 * v + 1]), pack_bf16x2(z[4 * v + 2], z[4 * v + 3]));
                    *reinterpret_cast<uint2*>(a.pieces + ((size_t)piece * s.T + t) * a.Ep + e) = r;
                    z[4 * v] -= bf16_lo(r.x); z[4 * v + 1] -= bf16_hi(r.x); z[4 * v + 2] -= bf16_lo(r.y); z[4 * v + 3] -= bf16_hi(r.y);
                }
            }
    }
    if constexpr (PRE) {
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
}

// dW_r on CTA pairs: 256 rows of dW_r x up to 256 experts, K = the tokens.  As in route_score_pair_kernel, what bounds such a product
// of three pieces is the traffic into shared memory, so a 64-token block of x (both operands lie with their columns contiguous) is
// fetched once and multiplied with that block of all three pieces; x and the pieces travel through separate rings; and the K loop
// is added up in segments of BW_SEG blocks, because the tensor core truncates where it adds.
//
// Few tiles, long sums: the token blocks of all tiles are laid in a row and cut into equal ranges, one for each pair.  A tile that one
// range covers goes to dW_r at once; of one that is cut, each range leaves its sums, and balance_sum_kernel adds them in order.
// T 16384, d 7168, E 256: 28 tiles of 256 blocks are 97 blocks for each pair (five equal ranges per tile made 104, and 140 sums).
// 122 us there, 180 GFLOP of issued products at 1.48 PFLOP/s: the tensor cores are busy for 84 % of a CTA's time, at 1.6 GHz.
// Two pieces would take a third less and keep 17 bits of dz: 2.4e-6 of dW_r's norm by calculation, where fp32 sums leave about 5e-7.
constexpr int BW_SA = 3, BW_SB = 9, BW_SLOT = 16384, BW_SEG = 3, BW_EPI_WARPS = 8;
constexpr int BW_THREADS = 64 + 32 * BW_EPI_WARPS;
constexpr int BW_SMEM_BYTES = (BW_SA + BW_SB) * BW_SLOT + BW_EPI_WARPS * ROW_STAGE_BYTES + 1024 /*align*/ + TC_BAR_BYTES;
// The row of token blocks in units of half a block of 256 experts (a last tile of at most 128 experts costs half): the tiles of 256
// experts, row tiles fastest, then the narrow ones.
struct BalCut {
    int tiles_m, wide, narrow, kb;        // row tiles, tiles of 256 experts, 0 or 1 narrow one, token blocks
    int range;                            // units of a pair
    __host__ __device__ int tiles() const { return tiles_m * (wide + narrow); }
    __host__ __device__ bool is_wide(int tile) const { return tile < tiles_m * wide; }
    __host__ __device__ int cost(int tile) const { return is_wide(tile) ? 2 * kb : kb; }
    __host__ __device__ int start(int tile) const {
        return is_wide(tile) ? tile * 2 * kb : tiles_m * wide * 2 * kb + (tile - tiles_m * wide) * kb;
    }
    __host__ __device__ int total() const { return start(tiles()); }
    __host__ __device__ int tile_at(int unit) const {
        const int w = tiles_m * wide * 2 * kb;
        return unit < w ? unit / (2 * kb) : tiles_m * wide + (unit - w) / kb;
    }
    __host__ __device__ int first_pair(int tile) const { return start(tile) / range; }
    __host__ __device__ int last_pair(int tile) const { return (start(tile) + cost(tile) - 1) / range; }
    // token block at which a unit of the tile lies (every block belongs to exactly one range)
    __host__ __device__ int block_at(int tile, int unit) const { return is_wide(tile) ? (unit - start(tile) + 1) / 2 : unit - start(tile); }
};
struct BalDwArgs {
    BalSeqs q;
    BalCut cut;
    int T, d, E;
    float* dW;
    float* part;           // [pairs][2][256][256]: sums of cut tiles, slot 0 of one that began in an earlier range, 1 of one that goes on
    int accumulate;
    int x_split;           // d is no multiple of 64: one copy per 64-wide chunk of x, whose edge is zero-filled
    int32_t* status;
    bool gemm_follows;
    PdlNote note;
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(BW_THREADS, 1)
bal_dw_pair_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmXe, const __grid_constant__ CUtensorMap tmP2,
                   const __grid_constant__ CUtensorMap tmP1, const BalDwArgs args) {
    extern __shared__ uint8_t tc_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tc_smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + (BW_SA + BW_SB) * BW_SLOT + BW_EPI_WARPS * ROW_STAGE_BYTES);
    // bars: fullA[SA] (leader's are used), emptyA[SA] (both), fullB[SB] (leader's), emptyB[SB] (both),
    //       tmem_full[2] (both), tmem_empty[2] (leader's)
    constexpr int NBARS = 2 * BW_SA + 2 * BW_SB + 4;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + NBARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = warp_index(), lane = threadIdx.x % 32;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const uint32_t smem_base = smem_u32(smem);
    const uint32_t bar_base = smem_u32(bars);
    auto fullA = [&](int s) { return bar_base + 8u * s; };
    auto emptyA = [&](int s) { return bar_base + 8u * (BW_SA + s); };
    auto fullB = [&](int s) { return bar_base + 8u * (2 * BW_SA + s); };
    auto emptyB = [&](int s) { return bar_base + 8u * (2 * BW_SA + BW_SB + s); };
    auto tfull_bar = [&](int b) { return bar_base + 8u * (2 * BW_SA + 2 * BW_SB + b); };
    auto tempty_bar = [&](int b) { return bar_base + 8u * (2 * BW_SA + 2 * BW_SB + 2 + b); };
    auto slotA = [&](int s) { return smem_base + (uint32_t)s * BW_SLOT; };
    auto slotB = [&](int s) { return smem_base + (uint32_t)(BW_SA + s) * BW_SLOT; };

    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * BW_SA + 2 * BW_SB; ++s) mbar_init(bar_base + 8u * s, 1);
        for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), 2 * BW_EPI_WARPS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch_desc(&tmX); tma_prefetch_desc(&tmXe); tma_prefetch_desc(&tmP2); tma_prefetch_desc(&tmP1);
    }
    if (warp == 1) tmem2_alloc(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();          // the peer's barriers exist before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    pdl_begin_gemm(args.gemm_follows, args.note);

    const int begin = bal_off(args.q, 0), end = bal_off(args.q, args.q.S);
    const int kb_first = begin / TC_BK, kblocks = end > begin ? (end - 1) / TC_BK + 1 - kb_first : 0;
    const BalCut cut = args.cut;
    const int pair = blockIdx.x >> 1;
    const int unit0 = min(cut.total(), pair * cut.range), unit1 = min(cut.total(), unit0 + cut.range);
    // columns of n-tile nt: 256, or 128 for a last tile of at most 128 columns
    auto tile_cols = [&](int nt) { return (args.E - 256 * nt <= 128) ? 128 : 256; };
    // the part of a tile that lies in this pair's range: rows of dW_r, experts, token blocks (of those that hold any tokens)
    struct Unit { int tile, mt, nt, kb0, kb1, next; };
    auto decode = [&](int unit) {
        Unit u;
        u.tile = cut.tile_at(unit);
        u.mt = u.tile % cut.tiles_m;
        u.nt = u.tile / cut.tiles_m;
        u.next = min(unit1, cut.start(u.tile) + cut.cost(u.tile));
        u.kb0 = max(kb_first, cut.block_at(u.tile, unit));
        u.kb1 = max(u.kb0, min(kb_first + kblocks, cut.block_at(u.tile, u.next)));
        return u;
    };

    if (warp == 0) {
        // ===================================================================== TMA producer (both CTAs)
        const bool el = elect_one();
        int sa = 0, sb = 0; uint32_t pa = 0, pb = 0; bool alive = true;
        for (int t = unit0, to; t < unit1 && alive; t = to) {
            const Unit u = decode(t);
            to = u.next;
            const int m0 = u.mt * 256 + 128 * (int)rank;          // past d: the copy fills zeros
            const int half_cols = tile_cols(u.nt) >> 1;           // this CTA's columns: 64 or 128
            const int chunk0 = (u.nt * 256 + (int)rank * half_cols) >> 6;
            const CUtensorMap* mp = half_cols == 128 ? &tmP2 : &tmP1;
            for (int kb = u.kb0; kb < u.kb1 && alive; ++kb) {
                if (!mbar_wait_all(emptyA(sa), pa ^ 1u, abort_flag, args.status, STATUS_WAIT_EMPTY)) { alive = false; break; }
                if (el) {
                    if (leader) mbar_expect_tx(fullA(sa), 2 * BW_SLOT);
                    const uint32_t fb = fullA(sa) & T2_PEER_MASK;
                    const bool dirty = bal_dirty(kb, begin, end, args.T);
                    const CUtensorMap* mx = dirty ? &tmXe : &tmX;
                    const int k0 = !dirty ? kb * TC_BK : kb == kb_first ? 0 : TC_BK;
                    if (!args.x_split) tma2_load_3d(slotA(sa), mx, fb, 0, k0, m0 >> 6);
                    else {
                        tma2_load_2d(slotA(sa), mx, fb, m0, k0);
                        tma2_load_2d(slotA(sa) + TC_CHUNK_BYTES, mx, fb, m0 + 64, k0);
                    }
                }
                if (++sa == BW_SA) { sa = 0; pa ^= 1u; }
                for (int ph = 0; ph < 3; ++ph) {
                    if (!mbar_wait_all(emptyB(sb), pb ^ 1u, abort_flag, args.status, STATUS_WAIT_EMPTY)) { alive = false; break; }
                    if (el) {
                        if (leader) mbar_expect_tx(fullB(sb), 2 * half_cols * TC_BK * 2);
                        // chunked map {64 columns, T rows, Ep/64 chunks, 3 pieces}
                        tma2_load_4d(slotB(sb), mp, fullB(sb) & T2_PEER_MASK, 0, kb * TC_BK, chunk0, ph);
                    }
                    if (++sb == BW_SB) { sb = 0; pb ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        // ===================================================================== MMA issuer (leader CTA)
        if (leader) {
            const bool el = elect_one();
            // kind::f16, bf16 x bf16 -> fp32, both operands with their columns contiguous, M = 256 over the pair; N per tile
            constexpr uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(256 >> 4) << 24);
            const uint64_t desc = smem_desc(0, TC_CHUNK_BYTES, 1024);
            constexpr uint32_t step = 2048 >> 4;        // 16 rows of K, 128 bytes each
            int sa = 0, sb = 0; uint32_t pa = 0, pb = 0; int it = 0; bool alive = true;
            for (int t = unit0, to; t < unit1 && alive; t = to) {
                const Unit u = decode(t);
                to = u.next;
                if (u.kb0 >= u.kb1) continue;
                const uint32_t idesc = idesc0 | ((uint32_t)(tile_cols(u.nt) >> 3) << 17);
                uint32_t d_tmem = 0;
                int kseg = BW_SEG;                       // K block inside the segment
                for (int kb = u.kb0; kb < u.kb1 && alive; ++kb) {
                    if (kseg == BW_SEG) {                // a new segment, in the other accumulator; the finished one goes to the epilogue
                        if (kb > u.kb0) {
                            if (el) umma2_commit_both(tfull_bar(it & 1));
                            ++it;
                        }
                        kseg = 0;
                        if (!mbar_wait_all(tempty_bar(it & 1), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, args.status,
                                           STATUS_WAIT_TMEM_EMPTY)) { alive = false; break; }
                        tc_fence_after();
                        d_tmem = tmem_base + (uint32_t)(it & 1) * TC_BN;
                    }
                    if (!mbar_wait_all(fullA(sa), pa, abort_flag, args.status, STATUS_WAIT_FULL)) { alive = false; break; }
                    const uint64_t da = desc | (uint64_t)((slotA(sa) & 0x3ffffu) >> 4);
                    for (int ph = 0; ph < 3; ++ph) {
                        if (!mbar_wait_all(fullB(sb), pb, abort_flag, args.status, STATUS_WAIT_FULL)) { alive = false; break; }
                        tc_fence_after();
                        const uint64_t db = desc | (uint64_t)((slotB(sb) & 0x3ffffu) >> 4);
                        if (el) {
#pragma unroll
                            for (int k4 = 0; k4 < TC_BK / 16; ++k4)
                                umma2_bf16(d_tmem, da + k4 * step, db + k4 * step, idesc, (kseg | ph | k4) != 0 ? 1u : 0u);
                            umma2_commit_both(emptyB(sb));
                        }
                        if (++sb == BW_SB) { sb = 0; pb ^= 1u; }
                    }
                    if (!alive) break;
                    if (el) umma2_commit_both(emptyA(sa));
                    if (++sa == BW_SA) { sa = 0; pa ^= 1u; }
                    ++kseg;
                }
                if (!alive) break;
                if (el) umma2_commit_both(tfull_bar(it & 1));
                ++it;
            }
        }
    } else {
        // ===================================================================== epilogue (8 warps, both CTAs)
        const int quarter = warp & 3;            // TMEM lanes 32*quarter .. +31 belong to this warp
        const int half = (warp - 2) >> 2;        // columns [128*half, 128*half + 128) of the tile
        int it = 0;
        bool ok = true;
        for (int t = unit0, to; t < unit1 && ok; t = to) {
            const Unit u = decode(t);
            to = u.next;
            const int nseg = (u.kb1 - u.kb0 + BW_SEG - 1) / BW_SEG;
            const bool active = half * 128 < tile_cols(u.nt);
            float sum[4][32];
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 32; ++i) sum[g][i] = 0.0f;
            for (int sg = 0; sg < nseg; ++sg) {
                const int b = it & 1;
                if (!mbar_wait_warp(tfull_bar(b), (uint32_t)(it >> 1) & 1u, abort_flag, args.status, STATUS_WAIT_TMEM_FULL,
                                    lane)) { ok = false; break; }
                tc_fence_after();
                if (active) {
                    const uint32_t ta = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)b * TC_BN + half * 128;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float part[32];
                        tmem_ld32(ta + 32 * g, part);
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[g][i] += part[i];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_pair(tempty_bar(b) & T2_PEER_MASK);
                ++it;
            }
            if (!ok) break;
            const int row0 = u.mt * 256 + 128 * (int)rank + quarter * 32, col = u.nt * 256 + half * 128;
            if (!active || row0 >= args.d) continue;
            const bool whole = cut.first_pair(u.tile) == cut.last_pair(u.tile);
            float* sh = reinterpret_cast<float*>(smem + (BW_SA + BW_SB) * BW_SLOT) + (warp - 2) * (ROW_STAGE_BYTES / 4);
            // (sums of a cut tile: rows of 256 columns, whatever the number of experts)
            float* out = whole ? args.dW + (size_t)row0 * args.E + col
                               : args.part + ((size_t)pair * 2 + (cut.first_pair(u.tile) < pair ? 0 : 1)) * 65536 +
                                     (size_t)(128 * (int)rank + quarter * 32) * 256 + half * 128;
            const size_t pitch = whole ? args.E : 256;
            const bool add = whole && args.accumulate;
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (col + 32 * g < args.E)
                    store_rows_32(sh, sum[g], out + 32 * g, pitch, min(32, args.d - row0), min(32, args.E - col - 32 * g), add, lane);
        }
    }

    // ------------------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) __nanosleep(1000);
        __syncthreads();
    }
    cluster_sync_all();          // neither CTA leaves while the other may still signal its barriers
    if (warp == 1) {
        tc_fence_after();
        tmem2_dealloc(tmem_base, 512);
    }
}

// The sums of the tiles that are cut, added in order, four experts a thread; and, by the blocks behind the first dw_blocks, the bias's
// gradient: 32 experts a block, its eight warps every eighth part.
struct BalSumArgs {
    BalCut cut;
    int d, E, dw_blocks;
    const float* part; float* dW;
    const float* dbias_part; float* dbias; int dbias_parts;
    int accumulate;
};
__global__ void __launch_bounds__(256) balance_sum_kernel(const BalSumArgs a) {
    pdl_begin();
    if ((int)blockIdx.x >= a.dw_blocks) {
        __shared__ float sh[8][32];
        const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, e = ((int)blockIdx.x - a.dw_blocks) * 32 + lane;
        float v = 0.0f;
        if (e < a.E)
#pragma unroll 8
            for (int b = warp; b < a.dbias_parts; b += 8) v += a.dbias_part[(size_t)b * a.E + e];
        sh[warp][lane] = v;
        __syncthreads();
        if (warp || e >= a.E) return;
        for (int w = 1; w < 8; ++w) v += sh[w][lane];
        a.dbias[e] = a.accumulate ? a.dbias[e] + v : v;
        return;
    }
    const int E4 = (a.E + 3) / 4;
    const size_t n = (size_t)a.d * E4;
    for (size_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)a.dw_blocks * 256) {
        const int row = (int)(i / E4), e = (int)(i - (size_t)row * E4) * 4;
        const int tile = (e >> 8) * a.cut.tiles_m + (row >> 8), p0 = a.cut.first_pair(tile), p1 = a.cut.last_pair(tile);
        if (p0 == p1) continue;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const float* at = a.part + (size_t)(row & 255) * 256 + (e & 255);
#pragma unroll 4
        for (int p = p0; p <= p1; ++p) {
            const float4 s = *reinterpret_cast<const float4*>(at + ((size_t)p * 2 + (p == p0 ? 1 : 0)) * 65536);
            v.x += s.x; v.y += s.y; v.z += s.z; v.w += s.w;
        }
        float* o = a.dW + (size_t)row * a.E + e;
        if (a.E % 4 == 0) {
            float4* o4 = reinterpret_cast<float4*>(o);
            if (a.accumulate) { v.x += o4->x; v.y += o4->y; v.z += o4->z; v.w += o4->w; }
            *o4 = v;
        } else {
            const float r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < a.E) o[j] = a.accumulate ? o[j] + r[j] : r[j];
        }
    }
}

// The same products on the CUDA cores, for contexts whose GEMMs run there (MOP_GEMM_SCALAR).
// dW_r = x^T dz over the tokens of the sequences; 64 x 64 outputs a block, 4 x 4 a thread.
__global__ void __launch_bounds__(256) balance_dw_kernel(const bf16* x, const float* dz, const BalSeqs q,
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
__global__ void __launch_bounds__(256) balance_dx_kernel(const float* dz, const float* W_r, const BalSeqs q,
                                                         bf16* __restrict__ dX, int T, int d, int E, int accumulate) {
    pdl_begin();
    __shared__ float sz[64][17], sw[64][17];
    const int i0 = blockIdx.y * 64, t0 = blockIdx.x * 64, tx = threadIdx.x % 16, ty = threadIdx.x / 16;
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
constexpr int BAL_PAIRS = 74;             // CTA pairs that the rules below count with (148 SMs)
inline int bal_warps(int E) { return E <= 512 ? 16 : 8; }
// Tokens per block of the forward: a single block where six rounds of its warps do (a second launch costs more), else two blocks for
// each SM, a round each at least.  The number of sequences does not enter, though a block takes 2 us for each of its own: T 1536, E 8
// (one block) 6.3, 15.5, 59 and 249 us with 1, 8, 32 and 128 sequences, T 1537 (seven) 9.1, 11, 19.5 and 49; T 4096, E 64 7.8, 8.5, 9.3 and 5.2.
inline int bal_chunk(int T, int E) {
    const int round = bal_warps(E) * (32 / bal_group(E)), c = (T + 295) / 296;
    return T <= 6 * round ? (T > 0 ? T : 1) : c < round ? round : c;
}
inline int bal_blocks(int T, int E) { return (T + bal_chunk(T, E) - 1) / bal_chunk(T, E); }
// ... of the backward: eight warps, one round of tokens for each of about 600 blocks.
inline int bal_chunk_bwd(int T, int E) {
    const int round = 8 * (E <= 64 ? 2 : 1), c = (T + 591) / 592;
    return c < round ? round : c;
}
inline int bal_blocks_bwd(int T, int E) { return (T + bal_chunk_bwd(T, E) - 1) / bal_chunk_bwd(T, E); }
inline size_t bal_smem_bytes(int E, int warps) { return (size_t)(warps + 1) * E * 4; }
inline BalShape bal_shape(const mop_moe_shape& s) {
    return {s.T, s.E, s.k, bal_group(s.E), s.score_fn, s.E % 4 == 0};
}
// Lanes per token in the backward: whole 64-wide blocks of experts, for the zeros behind the last one.
inline int bal_group_bwd(int E) { return E <= 64 ? 16 : 32; }
inline mop_status bal_init() {
    if (cudaFuncSetAttribute(bal_dw_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BW_SMEM_BYTES) != cudaSuccess) return MOP_ERR_CUDA;
    return vd_set_smem<VD_R, VD_PAIR>();
}
// Ranges of the dW_r product: equal shares of the row of token blocks, at least 8 blocks each, if that is worth the further launch and
// the sums' way to L2 and back (about 6 us) against whole tiles: a token block of 256 experts takes 0.8 us.
inline BalCut bal_cut(int T, int d, int E) {
    BalCut c{};
    const int rest = E % 256;
    c.tiles_m = (d + 255) / 256; c.kb = (T + 63) / 64;
    c.narrow = rest > 0 && rest <= 128 ? 1 : 0;
    c.wide = (E + 255) / 256 - c.narrow;
    const int most = c.wide ? 2 * c.kb : c.kb, per_block = c.wide ? 2 : 1, total = c.total();
    int share = (total + BAL_PAIRS - 1) / BAL_PAIRS;
    if (share < 8 * per_block) share = 8 * per_block;
    const int whole = (c.tiles() + BAL_PAIRS - 1) / BAL_PAIRS * most;
    c.range = (whole - share) * 0.4 > 6.0 ? share : whole;
    return c;
}
inline bool bal_is_cut(const BalCut& c) {
    for (int t = 0; t < c.tiles(); ++t)
        if (c.first_pair(t) != c.last_pair(t)) return true;
    return false;
}
constexpr size_t BAL_PART_BYTES = (size_t)BAL_PAIRS * 2 * 65536 * 4;
#define BAL_BY_WIDTH(E, GO)                                       \
    do {                                                          \
        if ((E) <= 128) GO(1);                                    \
        else if ((E) <= 256) GO(2);                               \
        else if ((E) <= 512) GO(4);                               \
        else GO(8);                                               \
    } while (0)

}  // namespace mop
