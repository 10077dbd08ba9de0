// Distillation from a teacher's top logits through the vocabulary projection (Eq. 5's projection with another loss on it):
//
//   Y = X W_voc (never stored),  s = Y / tau,  lse = log sum_v exp s_v,  q_k the teacher's probabilities of its K entries
//   loss[n] = sum_k q_k (log q_k - s[n, i_k] + lse[n])
//   dY[n,v] = dloss[n] / tau (Q p[n,v] - sum_{k: i_k = v} q_k),   p = exp(s - lse),   Q = sum_k q_k
//
// vd_gemm_kernel runs the products, with eight epilogue warps behind a TMA producer and an MMA issuer:
//   VD_L  Y = X W_voc: per row and up to 128 columns the maximum and the sum of exponentials, and the logits of the teacher's entries
//   VD_P  dY, one block of vocabulary columns, bf16 (the only piece of the N x V matrix that ever exists); with up to 128 rows two
//         pieces, dY = hi + lo
//   VD_X  dX = dY W_voc^T: the block's columns (its K) in `splits` ranges, fp32 sums over the blocks
//   VD_W  dW_voc[:, block] = X^T dY, bf16, beside VD_X
//   VD_R  the router's dX (+)= dz W_r^T (balance.cuh) from fp16 operands that are scaled by powers of two, bf16
// With many rows on CTA pairs (256 x 256 tiles, tcgen05.mma.cta_group::2, stages of 64 of K, as tc_gemm2_kernel).  With up to 128 rows
// a pair would multiply as much again in vain, and half of its stages would hold X: reading W is all there is then, and the product
// runs on single CTAs, tiles of 128 rows and up to 256 columns, whose rings hold as many bytes of W in flight as shared memory takes.
//
// One bf16 dY has an error of up to 2^-8 in each of its elements.  A row of dX is a sum over the vocabulary of its own token's dY, dW one
// over the tokens, and either way the errors add up as the terms do: they never average out, and with one piece the gradients are further
// off than their own rounding whatever the number of tokens.  Error over that of rounding them once, H 256, V 4096, K 5 and 64: dX as
// a whole 1.35 to 1.5 with 129, 300 and 2000 tokens alike, its worst row 2.3 to 2.7 (where one or two elements of dY outweigh the
// rest), dW 1.35 to 1.45; 1.1 to 1.9 where three tokens alone have a weight.  A second piece with what the first leaves out makes it 1.00,
// and doubles the two products behind it.  Up to 128 tokens these wait for W, and it costs 2 to 21 % (backward in us, one piece and two:
// N 10, H 1936, V 28800 86, 90; N 16, H 4096, V 64000 300, 305; N 64, H 2048, V 32000 100, 108; N 100, H 2048, V 50304 150, 170; N 128,
// H 7168, V 131072 1028, 1249).  Above, the tensor cores are the limit, and it would be more than half of the call again (N 1537,
// H 2048, V 50304: the two products are 249 and 220 of 870 us): one piece, as in mop_vocab_loss_bwd.
// Besides, VD_P sums its logits over all of H at once, where the tensor core truncates: 8e-6 of their size at H 7168, 2e-6 at 2048 (N 64; error of
// p 1.4e-5 with logits of 1.7, 6.9e-5 with logits of 8.5).  In dX that is nothing at the former and 1 % of its rounding at the latter.
//
// What bounds them, measured: many rows the tensor cores (VD_L N 2048, H 2048, V 32000 177 us, 1.52 PFLOP/s, where cuBLAS takes 180 for
// the same product with its bf16 store; N 8192, H 7168, V 131072 11.8 to 14.1 ms under the power cap, cuBLAS 11.1); few rows DRAM (VD_L
// N 64, H 2048, V 32000 27 us for 131 MB, 4.8 TB/s, against 30 us for a plain read of as many bytes; VD_W N 256 36 us for 131 MB of
// stores against 38 for a plain fill; VD_R T 16384, d 7168, E 256 69 us for 235 MB against 66).  Stores alone run at 3.6 to 3.9 TB/s on this part,
// so neither a deeper ring, nor more store boxes, nor evict-first lines, nor another tile order made VD_W or VD_R faster.
//
// A row's entries are sorted by column first (distill_prep_kernel), with the number of entries below each 64 columns beside them: the
// thread that owns the row fetches those of its columns while the tile is being multiplied.  VD_L on single CTAs waits long for its first
// tile: its warps read through the lists themselves, which saves the launch.
#pragma once
#include <limits.h>

#include "gemm_tc2.cuh"

namespace mop {

enum : int { VD_L = 0, VD_P = 1, VD_W = 2, VD_R = 3, VD_X = 4 };

// 32 rows, a lane each, of 32 fp32 columns to global memory: through shared memory (rows of 33), so that a warp's store is a row's 128
// bytes instead of 32 rows' 16 (a 256 x 256 tile's stores: about 4 us of the load-store unit's time with rows by lane, 0.6 this way).
constexpr int ROW_STAGE_BYTES = 32 * 33 * 4;
__device__ __forceinline__ void store_rows_32(float* sh, const float (&v)[32], float* out, size_t pitch, int rows, int cols, bool add, int lane) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) sh[lane * 33 + i] = v[i];
    __syncwarp();
    if (lane >= cols) return;
#pragma unroll 8
    for (int r = 0; r < rows; ++r) {
        float* o = out + r * pitch + lane;
        const float x = sh[r * 33 + lane];
        *o = add ? *o + x : x;
    }
}

// VD_PAIR; VD_ONE: single CTAs, rows up to 128; VD_HALF: up to 64, whose operand takes half the room (the instruction reads 128 rows
// all the same: what lies behind the 64 is the stage's own B, and what comes of it is not looked at).
enum : int { VD_PAIR = 0, VD_ONE = 1, VD_HALF = 2 };

// Stages, and store boxes (128 rows x 64 bf16 columns) for each column half: a tile fills two.  The router's product has a short
// main loop (its K are the experts), so its boxes are there twice: one pair is read by the copy engine while the next is filled.
template <int KIND, int MODE>
struct VdTraits {
    static constexpr bool PAIR = MODE == VD_PAIR;
    static constexpr bool STORES = KIND != VD_L && (PAIR || KIND != VD_X);       // (a single CTA's VD_X has two pieces to add up)
    static constexpr int SETS = KIND == VD_R ? 2 : 1;         // pairs of boxes
    static constexpr int BOXES = STORES ? 2 * SETS : 0;
    static constexpr int A_BYTES = MODE == VD_HALF ? T2_A_BYTES / 2 : T2_A_BYTES;
    static constexpr int RING_BYTES = PAIR ? (KIND == VD_L ? 6 : KIND == VD_R ? 3 : 5) * T2_STAGE_BYTES
                                           : (STORES ? 160 : 224) * 1024;
    static constexpr int STAGES = PAIR ? RING_BYTES / T2_STAGE_BYTES : 12;       // single CTAs: at most, as many as fit the tile's width
    static constexpr int SMEM_BYTES = RING_BYTES + 2 * BOXES * 16384 + 1024 /*align*/ + TC_BAR_BYTES;
    static int stages(int width) {
        const int fit = RING_BYTES / (PAIR ? T2_STAGE_BYTES : A_BYTES + width * TC_BK * 2);
        return fit < STAGES ? fit : STAGES;
    }
};
constexpr int VD_EPI_WARPS = 8;
constexpr int VD_THREADS = 64 + 32 * VD_EPI_WARPS;
constexpr int VD_BOX_BYTES = 128 * 64 * 2;
// K blocks (of 64) per accumulation segment of the forward.  The tensor core truncates where it adds; a segment starts from zero and
// the finished ones are added in fp32 registers, rounding to nearest.  Relative error of the logits at H 7168 2.5e-7 with 4, 4.8e-7 with 8
// (a plain fp32 product: 8.8e-7); N 2048, H 2048, V 32000 205 us with 4, 185 with 8, 183 with 16 or without segments.
constexpr int VD_SEG = 8;
constexpr int VD_MAX_K = 256;                                 // entries of a teacher's list

struct DistillLists {
    const int32_t* idx; const float* logits; const float* lse;      // the caller's: [N,K], [N,K], [N] or null
    int N, V, K;
    float tau;
};
struct VdArgs {
    int N, H, V, K;               // tokens, hidden size, vocabulary, entries per token
    int tiles_m, tiles_n, n_group, kblocks;
    int width, stages;            // columns of a tile, stages of the ring
    int n_base;                   // VD_P: first vocabulary column of the block
    int k_base;                   // VD_X: the same, added to W's K coordinate
    int cols;                     // columns of the whole output that exist
    int a_split, b_split;         // that operand's columns are no multiple of 64: one copy per 64-wide chunk, whose edge is zero-filled
    int piece_rows;               // dY has two pieces (maps of [2][N][columns]), of which a tile holds as many rows each: 64, 128, or 0: one
    int splits;                   // VD_X: ranges of K, as separate units of work (1 elsewhere)
    float c;                      // log2(e) / tau
    const int2* entry;            // [N, K] the row's entries by column (ascending): {column, place in the caller's list (VD_L) or dY (VD_P)}
    const uint16_t* first;        // [N, units + 1] how many of them lie below column 64 u
    int units;
    int parts;                    // VD_L: column ranges of `part`
    float* student;               // VD_L: [N, K] logits at the entries
    float2* part;                 // VD_L: [N, parts] (maximum, sum)
    DistillLists lists;           // VD_L on single CTAs, the first kernel of its call: the teacher's lists, and the status block, whose
    int32_t* clear;               // words it clears
    const float* coef;            // VD_P: dloss / tau Q per row
    const float* lse2;            // VD_P: log-sum-exp per row in units of log 2
    const float *row_scale, *col_scale;   // VD_R: what undoes the operands' scaling, per token and per 32 columns of dX
    bf16* add_to;                 // VD_R: dX [N, cols] that the product is added to, or null
    const int32_t* seq_off;       // VD_R: offsets of the sequences or null: rows outside [seq_off[0], seq_off[n_seq]) keep what they hold
    int n_seq;
    float* dx32;                  // VD_X: [splits (x 2 with two pieces), N, pitch] fp32 sums, or null (pairs only): one range and one block, dX is stored at once
    int pitch, accumulate;        // VD_X: add to them
    int32_t* status;
    bool gemm_follows;
    PdlNote note;
};

// "TMEM has been read": nothing in memory is published by it, so the arrival releases at CTA scope only.  (At cluster scope every
// arrival waits for the thread's own global stores first: the largest stall of the segmented loops.)
__device__ __forceinline__ void mbar_arrive_pair(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ float ex2(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The entries of a row in a range of columns, in ascending order: the next four are in registers.
struct VdEntries {
    const int2* list;
    int left;                     // entries that are not in registers yet
    int2 e[4];
    __device__ __forceinline__ void open(const VdArgs& a, int row, int col, int end, bool on) {       // whole units of 64
        left = 0;
        list = a.entry;
        if (on) {
            const uint16_t* f = a.first + (size_t)row * (a.units + 1);
            const int from = f[min(col >> 6, a.units)];
            left = (int)f[min(end >> 6, a.units)] - from;
            list = a.entry + (size_t)row * a.K + from;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) { e[i] = make_int2(INT_MAX, 0); if (i < left) e[i] = list[i]; }
        list += 4;
        left -= 4;
    }
    __device__ __forceinline__ int2 take() {
        const int2 r = e[0];
        e[0] = e[1]; e[1] = e[2]; e[2] = e[3];
        e[3] = make_int2(INT_MAX, 0);
        if (left > 0) { e[3] = *list; ++list; --left; }
        return r;
    }
};

// Eight values as bf16; what the rounding leaves out stays behind (nothing, where they are not finite).
__device__ __forceinline__ uint4 pack_and_keep_rest(float* v) {
    const uint4 r = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float rest = v[i] - (i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]));
        v[i] = fabsf(rest) < INFINITY ? rest : 0.0f;
    }
    return r;
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 :: "l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}

// The primitives on a pair (completing on, or signalling, both CTAs' or the leader's barriers) and on a single CTA.
template <bool PAIR>
__device__ __forceinline__ void vd_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
    if constexpr (PAIR) tma2_load_2d(dst, map, bar, x, y);
    else tma_load_2d(dst, map, bar, x, y);
}
template <bool PAIR>
__device__ __forceinline__ void vd_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
    if constexpr (PAIR) tma2_load_3d(dst, map, bar, x, y, z);
    else tma_load_3d(dst, map, bar, x, y, z);
}
template <bool PAIR>
__device__ __forceinline__ void vd_commit(uint32_t bar) {
    if constexpr (PAIR) umma2_commit_both(bar);
    else umma_commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void vd_arrive(uint32_t bar) {
    if constexpr (PAIR) mbar_arrive_pair(bar & T2_PEER_MASK);
    else mbar_arrive(bar);
}

// The same without the sorted lists: a warp goes through the lists of its 32 rows, lanes over the entries, sixteen loads in flight, and
// the thread that owns a row keeps the first eight entries of its columns (its offset, 7 bits, and its place in the list, 8 bits).
// Others are looked for again when they are wanted.
struct VdScan {
    const int32_t* list;
    int K, col, end, found;
    uint32_t e[4];
    __device__ __forceinline__ void open(const DistillLists& l, int row0, int rows, int from, int to, int lane) {
        K = l.K; col = from; end = min(to, l.V); found = 0;
        list = l.idx + (size_t)(row0 + lane) * K;
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = 0;
        const int words = (K + 31) / 32, n = rows * words;                // word w of row r: its entries 32 w + lane
        const int32_t* base = l.idx + (size_t)row0 * K;
        int r = 0, w = 0, rr = 0, ww = 0;                                 // of the next load, and of the next word that is looked at
        for (int i0 = 0; i0 < n; i0 += 16) {
            int v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[i] = i0 + i < n && 32 * w + lane < K ? base[(size_t)r * K + 32 * w + lane] : -1;
                if (++w == words) { w = 0; ++r; }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                uint32_t hits = __ballot_sync(0xffffffffu, v[i] >= col && v[i] < end);
                while (hits) {
                    const int b = __ffs(hits) - 1;
                    hits &= hits - 1;
                    const int c = __shfl_sync(0xffffffffu, v[i], b);
                    if (lane != rr) continue;
                    const uint32_t packed = (uint32_t)(c - col) | (uint32_t)(32 * ww + b) << 7;
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (found == q) e[q / 2] |= packed << 16 * (q % 2);
                    ++found;
                }
                if (++ww == words) { ww = 0; ++rr; }
            }
        }
    }
    template <class F>            // f(offset of the column, place in the list)
    __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < found) f((int)(e[i / 2] >> 16 * (i % 2) & 127u), (int)(e[i / 2] >> (16 * (i % 2) + 7) & 255u));
        if (found <= 8) return;
        int seen = 0;
        for (int k0 = 0; k0 < K; k0 += 8) {
            int v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k0 + i < K ? list[k0 + i] : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] >= col && v[i] < end && ++seen > 8) f(v[i] - col, k0 + i);
        }
    }
};

template <int KIND, int MODE>
__global__ void __cluster_dims__(MODE == VD_PAIR ? 2 : 1, 1, 1) __launch_bounds__(VD_THREADS, 1)
vd_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmO,
               const VdArgs args) {
    using Tr = VdTraits<KIND, MODE>;
    constexpr bool PAIR = Tr::PAIR;
    static_assert(PAIR || KIND == VD_L || KIND == VD_P || (KIND == VD_X && MODE == VD_ONE), "the kinds whose rows are few tokens");
    constexpr int S = Tr::STAGES;
    constexpr int TM = PAIR ? 256 : 128;
    constexpr bool A_MN = KIND == VD_W;                       // the tokens are K: X^T lies with M contiguous
    constexpr bool B_MN = KIND != VD_R && KIND != VD_X;
    extern __shared__ uint8_t tc_smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(tc_smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* boxes = smem + Tr::RING_BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(boxes + 2 * Tr::BOXES * VD_BOX_BYTES);
    // bars: [0,S) full (leader's are used), [S,2S) empty (both), tmem_full[2] (both), tmem_empty[2] (leader's)
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * S + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = warp_index(), lane = threadIdx.x % 32;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const bool leader = rank == 0;
    const uint32_t smem_base = smem_u32(smem);
    const uint32_t bar_base = smem_u32(bars);
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (S + s); };
    auto tfull_bar = [&](int b) { return bar_base + 8u * (2 * S + b); };
    auto tempty_bar = [&](int b) { return bar_base + 8u * (2 * S + 2 + b); };

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(tfull_bar(b), 1); mbar_init(tempty_bar(b), (PAIR ? 2 : 1) * VD_EPI_WARPS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        tma_prefetch_desc(&tmA); tma_prefetch_desc(&tmB);
        if (Tr::STORES) tma_prefetch_desc(&tmO);
    }
    if (warp == 1) {
        if constexpr (PAIR) tmem2_alloc(smem_u32(tmem_slot), 512);
        else tmem_alloc(smem_u32(tmem_slot), 512);
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();      // the peer's barriers exist before anything signals them
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    // The weight gradient runs beside dX of its block, the router's dX beside its weight gradient: both read the logit gradients, neither
    // what the other writes.
    constexpr bool BESIDE = KIND == VD_W || KIND == VD_R;
    const bool beside = BESIDE && args.note.word;
    if (beside) pdl_begin_beside(args.gemm_follows, args.note);
    else pdl_begin_gemm(args.gemm_follows, args.note);
    if constexpr (!PAIR && KIND == VD_L)
        if (args.clear && blockIdx.x == 0 && threadIdx.x == 0) { args.clear[0] = 0; args.clear[VOCAB_NOTE] = 0; }     // (a wait runs out after seconds)

    const int tiles = args.tiles_m * args.tiles_n, total = KIND == VD_X ? tiles * args.splits : tiles;
    const int cluster_id = PAIR ? blockIdx.x >> 1 : blockIdx.x, n_clusters = PAIR ? gridDim.x >> 1 : gridDim.x;
    // a pair's CTAs hold half of the tile's columns each
    const int width = PAIR && (KIND == VD_W || KIND == VD_R || KIND == VD_X) ? 256 : args.width, my_cols = PAIR ? width / 2 : width;
    const int stages = PAIR ? S : args.stages;
    const uint32_t stage_bytes = PAIR ? T2_STAGE_BYTES : Tr::A_BYTES + my_cols * TC_BK * 2;
    const uint32_t copy_bytes = Tr::A_BYTES + my_cols * TC_BK * 2;
    // blocks of n_group n-tiles, row tiles slower inside one: the pairs that run at the same time cover a nearly square patch
    auto decode = [&](int t, int& mt, int& nt, int& kb0, int& kb1) {
        kb0 = 0; kb1 = args.kblocks;
        if constexpr (KIND == VD_X) {
            const int ks = t / tiles, q = args.kblocks / args.splits, r = args.kblocks - q * args.splits;
            t -= ks * tiles;
            kb0 = ks * q + min(ks, r);
            kb1 = kb0 + q + (ks < r ? 1 : 0);
        }
        const int per = args.n_group * args.tiles_m, g = t / per, r = t - g * per;
        const int w = min(args.n_group, args.tiles_n - g * args.n_group);
        mt = r / w;
        nt = g * args.n_group + r - mt * w;
    };

    if (warp == 0) {
        // ===================================================================== TMA producer (both CTAs)
        const bool el = elect_one();
        int stage = 0; uint32_t phase = 0; bool alive = true;
        for (int t = cluster_id; t < total && alive; t += n_clusters) {
            int mt, nt, kb0, kb1;
            decode(t, mt, nt, kb0, kb1);
            const int m0 = TM * mt + 128 * (int)rank, n0 = args.n_base + width * nt + my_cols * (int)rank;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait_all(empty_bar(stage), phase ^ 1u, abort_flag, args.status, STATUS_WAIT_EMPTY)) { alive = false; break; }
                const uint32_t fb = PAIR ? full_bar(stage) & T2_PEER_MASK : full_bar(stage);      // the leader's barrier
                const uint32_t sA = smem_base + stage * stage_bytes, sB = sA + Tr::A_BYTES;
                const int k0 = kb * TC_BK;
                if (el) {
                    if (leader) mbar_expect_tx(full_bar(stage), (PAIR ? 2 : 1) * copy_bytes);
                    // two pieces: the same tokens of X against both; both pieces' rows as the rows of dX's tile
                    const int ka = KIND == VD_W && args.piece_rows ? k0 % args.piece_rows : k0;
                    if (KIND == VD_X && args.piece_rows) vd_load_3d<PAIR>(sA, &tmA, fb, k0, 0, (int)rank);
                    else if constexpr (!A_MN) vd_load_2d<PAIR>(sA, &tmA, fb, k0, m0);
                    else if (!args.a_split) vd_load_3d<PAIR>(sA, &tmA, fb, 0, ka, m0 >> 6);
                    else {
                        vd_load_2d<PAIR>(sA, &tmA, fb, m0, ka);
                        vd_load_2d<PAIR>(sA + TC_CHUNK_BYTES, &tmA, fb, m0 + 64, ka);
                    }
                    if (KIND == VD_W && args.piece_rows) tma2_load_4d(sB, &tmB, fb, 0, ka, n0 >> 6, k0 / args.piece_rows);
                    else if constexpr (!B_MN) vd_load_2d<PAIR>(sB, &tmB, fb, k0 + (KIND == VD_X ? args.k_base : 0), n0);
                    else if (!args.b_split) vd_load_3d<PAIR>(sB, &tmB, fb, 0, k0, n0 >> 6);
                    else
                        for (int q = 0; q < my_cols; q += 64) vd_load_2d<PAIR>(sB + q * (TC_CHUNK_BYTES / 64), &tmB, fb, n0 + q, k0);
                }
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else if (warp == 1) {
        // ===================================================================== MMA issuer (leader CTA)
        if (leader) {
            const bool el = elect_one();
            // VD_R: both operands fp16 (format 0) instead of bf16 (1)
            const uint32_t idesc = (((PAIR ? make_idesc2(A_MN, B_MN) : make_idesc(A_MN, B_MN)) & (KIND == VD_R ? ~((1u << 7) | (1u << 10)) : ~0u)) &
                                    ~(63u << 17)) | ((uint32_t)(width >> 3) << 17);
            const uint64_t desc_a = A_MN ? smem_desc(0, TC_CHUNK_BYTES, 1024) : smem_desc(0, 0, 1024);
            const uint64_t desc_b = B_MN ? smem_desc(0, TC_CHUNK_BYTES, 1024) : smem_desc(0, 0, 1024);
            constexpr uint32_t a_step = (A_MN ? 2048 : 32) >> 4, b_step = (B_MN ? 2048 : 32) >> 4;
            int stage = 0; uint32_t phase = 0; int it = 0; bool alive = true;
            for (int t = cluster_id; t < total && alive; t += n_clusters) {
                int mt, nt, kb0, kb1;
                decode(t, mt, nt, kb0, kb1);
                uint32_t d_tmem = 0;
                int kseg = 0;                            // K block inside the segment
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (kb == kb0 || (KIND == VD_L && kseg == VD_SEG)) {
                        if (kb > kb0) {                        // segment done: the epilogue adds it up, the next one goes to the other accumulator
                            if (el) vd_commit<PAIR>(tfull_bar(it & 1));
                            ++it;
                            kseg = 0;
                        }
                        if (!mbar_wait_all(tempty_bar(it & 1), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, args.status,
                                           STATUS_WAIT_TMEM_EMPTY)) { alive = false; break; }
                        tc_fence_after();
                        d_tmem = tmem_base + (uint32_t)(it & 1) * TC_BN;
                    }
                    if (!mbar_wait_all(full_bar(stage), phase, abort_flag, args.status, STATUS_WAIT_FULL)) { alive = false; break; }
                    tc_fence_after();
                    const uint32_t sA = smem_base + stage * stage_bytes;
                    const uint64_t da = desc_a | (uint64_t)((sA & 0x3ffffu) >> 4);
                    const uint64_t db = desc_b | (uint64_t)(((sA + Tr::A_BYTES) & 0x3ffffu) >> 4);
                    if (el) {
#pragma unroll
                        for (int k4 = 0; k4 < TC_BK / 16; ++k4) {
                            if constexpr (PAIR) umma2_bf16(d_tmem, da + k4 * a_step, db + k4 * b_step, idesc, (kseg | k4) != 0 ? 1u : 0u);
                            else umma_bf16(d_tmem, da + k4 * a_step, db + k4 * b_step, idesc, (kseg | k4) != 0 ? 1u : 0u);
                        }
                        vd_commit<PAIR>(empty_bar(stage));
                    }
                    ++kseg;
                    if (++stage == stages) { stage = 0; phase ^= 1u; }
                }
                if (!alive) break;
                if (el) vd_commit<PAIR>(tfull_bar(it & 1));
                ++it;
            }
        }
    } else {
        // ===================================================================== epilogue (8 warps, both CTAs)
        const int quarter = warp & 3;            // TMEM lanes 32*quarter .. +31 belong to this warp
        const int half = (warp - 2) >> 2;        // columns [128*half, 128*half + 128) of the tile
        const uint32_t ta0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + half * 128;
        int it = 0;
        bool ok = true;
        for (int t = cluster_id; t < total && ok; t += n_clusters) {
            int mt, nt, kb0, kb1;
            decode(t, mt, nt, kb0, kb1);
            const int row = TM * mt + 128 * (int)rank + quarter * 32 + lane;
            const int col0 = args.n_base + width * nt + 128 * half;       // this thread's first column of the output
            const int tile_end = args.n_base + width * (nt + 1);          // (a half behind it has no columns)
            if constexpr (KIND == VD_L) {
                const bool mine = row < args.N;
                VdEntries en;
                VdScan scan;
                (void)en; (void)scan;
                if constexpr (PAIR) en.open(args, row, col0, min(col0 + 128, tile_end), mine && col0 < tile_end);
                else scan.open(args.lists, quarter * 32, col0 < tile_end ? min(32, max(0, args.N - quarter * 32)) : 0, col0, min(col0 + 128, tile_end), lane);
                float y[4][32];
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[g][i] = 0.0f;
                const int nseg = (kb1 + VD_SEG - 1) / VD_SEG;
                for (int sg = 0; sg < nseg; ++sg) {
                    if (!mbar_wait_warp(tfull_bar(it & 1), (uint32_t)(it >> 1) & 1u, abort_flag, args.status, STATUS_WAIT_TMEM_FULL,
                                        lane)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float part[32];
                        tmem_ld32(ta0 + (uint32_t)(it & 1) * TC_BN + 32 * g, part);
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[g][i] += part[i];
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) vd_arrive<PAIR>(tempty_bar(it & 1));
                    ++it;
                }
                if (!ok) break;
                float m = -INFINITY, sum = 0.0f;
                const int end = min(args.cols, tile_end);
                if (col0 + 128 > end) {                   // the vocabulary, or the tile, ends inside these columns
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (col0 + 32 * g + i >= end) y[g][i] = -INFINITY;
                }
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int i = 0; i < 32; ++i) m = fmaxf(m, y[g][i]);
                const float mc = m == -INFINITY ? 0.0f : m * args.c;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum += ex2(fmaf(y[g][i], args.c, -mc));
                    if constexpr (PAIR)
                        while (en.e[0].x < col0 + 32 * (g + 1)) {         // (entries lie inside the vocabulary)
                            const int2 e = en.take();
                            const int i = e.x - col0 - 32 * g;
                            float v = 0.0f;
#pragma unroll
                            for (int q = 0; q < 32; ++q) v = i == q ? y[g][q] : v;
                            args.student[(size_t)row * args.K + e.y] = v;
                        }
                }
                if constexpr (!PAIR)
                    scan.each([&](int at, int k) {
                        float v = 0.0f;
#pragma unroll
                        for (int g = 0; g < 4; ++g)
#pragma unroll
                            for (int q = 0; q < 32; ++q) v = at == 32 * g + q ? y[g][q] : v;
                        args.student[(size_t)row * args.K + k] = v;
                    });
                if (mine && col0 < tile_end) args.part[(size_t)row * args.parts + (width > 128 ? 2 * nt + half : nt)] = make_float2(m, sum);
            } else {
                const bool mine = row < args.N;
                float coef = 0.0f, lse2 = 0.0f;
                bool inside = true, padding = false;
                float scale[4] = {};
                (void)scale; (void)padding;
                if constexpr (KIND == VD_R) {
                    if (mine) coef = args.row_scale[row];
#pragma unroll
                    for (int g = 0; g < 4; ++g) scale[g] = args.col_scale[col0 / 32 + g];
                    if (args.seq_off) {
                        const int begin = args.seq_off[0], end = args.seq_off[args.n_seq], r0 = row - (quarter * 32 + lane);
                        inside = row >= begin && row < end;
                        padding = r0 < begin || min(r0 + 128, args.N) > end;       // among the CTA's 128 rows
                    }
                }
                VdEntries en;
                (void)en;
                if constexpr (KIND == VD_P) {
                    if (mine) { coef = args.coef[row]; lse2 = args.lse2[row]; }
                    en.open(args, row, col0, min(col0 + 128, tile_end), mine && col0 < tile_end);
                }
                bool ready = mbar_wait_warp(tfull_bar(it & 1), (uint32_t)(it >> 1) & 1u, abort_flag, args.status, STATUS_WAIT_TMEM_FULL, lane);
                // the four warps of a column half meet at named barriers below: they give up together or not at all
                if (!bar_vote_all(1 + half, 128, ready)) { ok = false; break; }
                tc_fence_after();
                float y[4][32];
                (void)inside;
                const uint32_t ta = ta0 + (uint32_t)(it & 1) * TC_BN;
                tmem_ld32_nowait(ta, y[0]);
                tmem_ld32_nowait(ta + 32, y[1]);
                tmem_ld32_nowait(ta + 64, y[2]);
                tmem_ld32_nowait(ta + 96, y[3]);
                tmem_ld_wait4(y[0], y[1], y[2], y[3]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) vd_arrive<PAIR>(tempty_bar(it & 1));
                ++it;
                if constexpr (KIND == VD_X)
                    if (!Tr::STORES || args.dx32) {
                        const int piece = args.piece_rows ? (row - lane) / args.piece_rows : 0, row0 = row - lane - piece * args.piece_rows;
                        float* out = args.dx32 + ((size_t)(t / tiles * (args.piece_rows ? 2 : 1) + piece) * args.N + row0) * args.pitch + col0;
                        float* sh = reinterpret_cast<float*>(boxes) + (warp - 2) * (ROW_STAGE_BYTES / 4);    // (pairs: the boxes' room)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            if (col0 + 32 * g >= min(args.pitch, tile_end)) continue;
                            if constexpr (PAIR) store_rows_32(sh, y[g], out + 32 * g, args.pitch, min(32, args.N - row0), 32, args.accumulate != 0, lane);
                            else if (row0 + lane < args.N) epi_f32<32>(out + (size_t)lane * args.pitch + 32 * g, y[g], args.accumulate);
                        }
                        continue;
                    }
                const bool issuer = quarter == 0 && lane == 0;
                const int set = Tr::SETS == 2 ? (it - 1) & 1 : 0;
                uint8_t* box = boxes + (Tr::BOXES * half + 2 * set) * VD_BOX_BYTES;
                if constexpr (KIND == VD_P) {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[g][i] = coef * ex2(fmaf(y[g][i], args.c, -lse2));
                }
                if constexpr (KIND == VD_R) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        scale[g] *= coef;
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[g][i] *= scale[g];
                    }
                    if (padding && !inside)               // (0 times a router weight that is not finite)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
#pragma unroll
                            for (int i = 0; i < 32; ++i) y[g][i] = 0.0f;
                    if (args.add_to && mine && inside) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            if (col0 + 8 * j >= args.cols) continue;
                            float* v = &y[j / 4][(j % 4) * 8];
                            const uint4 o = *reinterpret_cast<const uint4*>(args.add_to + (size_t)row * args.cols + col0 + 8 * j);
                            v[0] += bf16_lo(o.x); v[1] += bf16_hi(o.x); v[2] += bf16_lo(o.y); v[3] += bf16_hi(o.y);
                            v[4] += bf16_lo(o.z); v[5] += bf16_hi(o.z); v[6] += bf16_lo(o.w); v[7] += bf16_hi(o.w);
                        }
                    }
                    // Where padding is to stay as it is, a box with some of it is written by rows: a copy of the box would read and
                    // write it again, and a NaN in it would not keep its bits.
                    if (args.add_to && padding) {
                        if (mine && inside)
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                if (col0 + 8 * j >= args.cols) continue;
                                const float* v = &y[j / 4][(j % 4) * 8];
                                *reinterpret_cast<uint4*>(args.add_to + (size_t)row * args.cols + col0 + 8 * j) =
                                    make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                            }
                        if (issuer) tma_store_commit();       // (an empty group: the box sets are told apart by counting groups)
                        continue;
                    }
                }
                if constexpr (KIND == VD_P && !PAIR) {    // the teacher's entries, and two pieces: 64 rows of each in a box, or 128 in turn
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        while (en.e[0].x < col0 + 32 * (g + 1)) {
                            const int2 e = en.take();
#pragma unroll
                            for (int q = 0; q < 32; ++q) y[g][q] = e.x - col0 - 32 * g == q ? __int_as_float(e.y) : y[g][q];
                        }
#pragma unroll
                    for (int piece = 0; piece < (MODE == VD_ONE ? 2 : 1); ++piece) {
                        if (issuer) tma_store_wait_read<0>();
                        asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
                        if (MODE == VD_ONE || quarter < 2) {
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                uint8_t* rowp = box + h * VD_BOX_BYTES + (quarter * 32 + lane) * 128;
#pragma unroll
                                for (int j = 0; j < 8; ++j) {
                                    float* v = &y[2 * h + j / 4][(j % 4) * 8];
                                    uint8_t* at = rowp + ((j ^ (lane & 7)) << 4);
                                    *reinterpret_cast<uint4*>(at) = pack_and_keep_rest(v);
                                    if (MODE == VD_HALF) *reinterpret_cast<uint4*>(at + VD_BOX_BYTES / 2) = pack_and_keep_rest(v);
                                }
                            }
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
                        if (issuer) {
                            const int x = width * nt + 128 * half, end = min(args.cols, width * (nt + 1));
                            if (x < end) tma_store_3d(&tmO, smem_u32(box), x, 0, piece);
                            if (x + 64 < end) tma_store_3d(&tmO, smem_u32(box + VD_BOX_BYTES), x + 64, 0, piece);
                            tma_store_commit();
                        }
                    }
                    continue;
                }
                if (issuer) tma_store_wait_read<Tr::SETS - 1>();          // this pair's last copies have been read
                asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
#pragma unroll
                for (int h = 0; h < 2; ++h) {             // boxes of 128-byte rows, 16-byte chunks swizzled by row
                    uint8_t* rowp = box + h * VD_BOX_BYTES + (quarter * 32 + lane) * 128;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float* v = &y[2 * h + j / 4][(j % 4) * 8];
                        *reinterpret_cast<uint4*>(rowp + ((j ^ (lane & 7)) << 4)) =
                            make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                    }
                    if constexpr (KIND == VD_P)
                        while (en.e[0].x < col0 + 64 * (h + 1)) {         // the teacher's entries among these columns
                            const int2 e = en.take();
                            const int i = e.x - col0 - 64 * h;
                            *reinterpret_cast<bf16*>(rowp + (((i >> 3) ^ (lane & 7)) << 4) + (i & 7) * 2) =
                                __float2bfloat16_rn(__int_as_float(e.y));
                        }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
                if (issuer) {
                    const int x = width * nt + 128 * half, r0 = TM * mt + 128 * (int)rank, end = min(args.cols, width * (nt + 1));
                    if (r0 < (KIND == VD_W ? args.H : args.N)) {
                        if (x < end) tma_store_2d(&tmO, smem_u32(box), x, r0);
                        if (x + 64 < end) tma_store_2d(&tmO, smem_u32(box + VD_BOX_BYTES), x + 64, r0);
                    }
                    tma_store_commit();
                }
            }
        }
        if (Tr::STORES && quarter == 0 && lane == 0) tma_store_wait_all();       // boxes read, and written, before the CTA exits
    }

    // ------------------------------------------------------------------------- teardown
    if (beside) pdl_end_beside();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) __nanosleep(1000);
        __syncthreads();
    }
    if constexpr (PAIR) cluster_sync_all();      // neither CTA leaves while the other may still signal its barriers
    if (warp == 1) {
        tc_fence_after();
        if constexpr (PAIR) tmem2_dealloc(tmem_base, 512);
        else tmem_dealloc(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------ the teacher's lists
// Teacher's probabilities of the entries lane + 32 j of row n (0 where there is none), and log q; a row without entries has none.
template <int J>
__device__ __forceinline__ void distill_teacher(const DistillLists& l, size_t n, int lane, int32_t (&col)[J], float (&q)[J], float (&logq)[J]) {
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int k = lane + 32 * j;
        col[j] = INT_MAX;
        logq[j] = -INFINITY;
        if (k < l.K) {
            const int32_t v = l.idx[n * l.K + k];
            if (v >= 0 && v < l.V) { col[j] = v; logq[j] = __fdiv_rn(l.logits[n * l.K + k], l.tau); }
        }
        m = fmaxf(m, logq[j]);
    }
    float norm = 0.0f;
    if (l.lse) {
        norm = l.lse[n];
    } else {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (m == -INFINITY) m = 0.0f;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) s += expf(logq[j] - m);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        norm = s == 0.0f ? 0.0f : m + logf(s);
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (col[j] != INT_MAX) logq[j] -= norm;
        q[j] = col[j] != INT_MAX ? expf(logq[j]) : 0.0f;
    }
}

struct DistillPrep {
    DistillLists l;
    int2* entry; uint16_t* first; int units;                        // as in VdArgs
    const float* student; const float* lse; const float* dloss;     // backward
    float* coef; float* lse2;
    int32_t* status;
};
constexpr int DP_WARPS = 8;
// 18 us forward and 24 backward for 8044 rows of 97 entries (38 and 54 when each entry counted the smaller ones).
// A warp per row: sorts the entries by column (equal columns by their place in the list; those outside the vocabulary last) in registers,
// entry 32 j + lane with lane, a bitonic network.  Backward: dY of each entry, the probabilities of equal columns added up, so that
// every one of them holds the same value.
template <int J, bool BWD>
__global__ void __launch_bounds__(32 * DP_WARPS) distill_prep_kernel(const DistillPrep a) {
    pdl_begin();
    __shared__ int32_t scols[DP_WARPS][32 * J];
    __shared__ float sq[DP_WARPS][BWD ? 32 * J : 1], sorted_q[DP_WARPS][BWD ? 32 * J : 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, N = a.l.N, K = a.l.K;
    if (blockIdx.x == 0 && threadIdx.x == 0) { *a.status = 0; a.status[VOCAB_NOTE] = 0; }
    for (int n = blockIdx.x * DP_WARPS + warp; n < N; n += gridDim.x * DP_WARPS) {
        int32_t col[J];
        float q[J], logq[J];
        float total = 0.0f, g = 0.0f, lse = 0.0f;
        if constexpr (BWD) {
            g = __fdiv_rn(a.dloss[n], a.l.tau);
            lse = a.lse[n];
            distill_teacher<J>(a.l, n, lane, col, q, logq);
#pragma unroll
            for (int j = 0; j < J; ++j) total += q[j];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
            if (lane == 0) { a.coef[n] = g * total; a.lse2[n] = lse * 1.4426950408889634f; }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < J; ++j) sq[warp][lane + 32 * j] = q[j];
        } else {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const int k = lane + 32 * j;
                const int32_t v = k < K ? a.l.idx[(size_t)n * K + k] : -1;
                col[j] = v >= 0 && v < a.l.V ? v : INT_MAX;
            }
        }
        unsigned long long key[J];
#pragma unroll
        for (int j = 0; j < J; ++j) key[j] = (unsigned long long)(uint32_t)col[j] << 8 | (uint32_t)(lane + 32 * j);
#pragma unroll
        for (int size = 2; size <= 32 * J; size *= 2)
#pragma unroll
            for (int step = size / 2; step > 0; step /= 2)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const bool up = ((lane + 32 * j) & size) == 0;        // this run ascends
                    if (step >= 32) {
                        const int o = j ^ (step / 32);
                        if (o > j && (key[j] > key[o]) == up) { const unsigned long long t = key[j]; key[j] = key[o]; key[o] = t; }
                    } else {
                        const unsigned long long other = __shfl_xor_sync(0xffffffffu, key[j], step);
                        const bool low = (lane & step) == 0;
                        if ((key[j] > other) == (up == low)) key[j] = other;
                    }
                }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int32_t c = (int32_t)(key[j] >> 8);
            scols[warp][lane + 32 * j] = c;
            if constexpr (BWD) sorted_q[warp][lane + 32 * j] = sq[warp][key[j] & 255];
        }
        __syncwarp();
        int valid = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = lane + 32 * j, k = (int)(key[j] & 255);
            const int32_t c = (int32_t)(key[j] >> 8);
            valid += __popc(__ballot_sync(0xffffffffu, c != INT_MAX));
            if (at >= K) continue;
            int2 e = make_int2(c, k);
            if (c != INT_MAX) {
                if constexpr (BWD) {
                    int from = at;
                    while (from > 0 && scols[warp][from - 1] == c) --from;
                    float same = 0.0f;
                    for (; from < 32 * J && scols[warp][from] == c; ++from) same += sorted_q[warp][from];
                    const float p = expf(__fdiv_rn(a.student[(size_t)n * K + k], a.l.tau) - lse);
                    e.y = __float_as_int(g * fmaf(total, p, -same));
                }
                // the columns' units up to this entry's, from the one behind the entry before it
                for (int u = at > 0 ? (scols[warp][at - 1] >> 6) + 1 : 0; u <= c >> 6; ++u)
                    a.first[(size_t)n * (a.units + 1) + u] = (uint16_t)at;
            }
            a.entry[(size_t)n * K + at] = e;
        }
        for (int u = (valid > 0 ? (scols[warp][valid - 1] >> 6) + 1 : 0) + lane; u <= a.units; u += 32)
            a.first[(size_t)n * (a.units + 1) + u] = (uint16_t)valid;
    }
}

// lse of a row from its (maximum, sum) pairs, R warps over the pairs; then the loss, the first warp's lanes over the entries, whose
// values it has fetched before.  Four warps a row where there are few rows or long ones, else one (8044 rows of 192 pairs, 97 entries: 32
// us with four, 14 with one; 64 rows of 250 pairs: 18 us with a block of eight warps for 32 rows, 5 with four for each).
struct DistillMerge {
    DistillLists l;
    const float2* part; int parts;
    float* student;
    float c;
    float *loss, *lse;
};
constexpr int DM_THREADS = 128;
template <int J, int R>
__global__ void __launch_bounds__(DM_THREADS) distill_merge_kernel(const DistillMerge a) {
    pdl_begin();
    __shared__ float sh[2][R];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32 % R, tid = warp * 32 + lane, K = a.l.K;
    const size_t n = R == 1 ? (size_t)blockIdx.x * (DM_THREADS / 32) + threadIdx.x / 32 : blockIdx.x;
    if (n >= a.l.N) return;                               // (whole warps, and with R > 1 no block has any)
    const float2* row = a.part + n * a.parts;
    constexpr int HELD = R == 1 ? 8 : 4;                  // pairs of a thread that stay in registers
    float2 v[HELD];
    float m = -INFINITY, t = 0.0f;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        v[i] = make_float2(-INFINITY, 0.0f);
        if (tid + i * 32 * R < a.parts) v[i] = row[tid + i * 32 * R];
        m = fmaxf(m, v[i].x);
    }
    for (int i = tid + HELD * 32 * R; i < a.parts; i += 32 * R) m = fmaxf(m, row[i].x);
    int32_t col[J];
    float q[J], logq[J], s[J];
    if (warp == 0) {
        distill_teacher<J>(a.l, n, lane, col, q, logq);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            s[j] = 0.0f;
            if (lane + 32 * j >= K) continue;
            if (col[j] != INT_MAX) s[j] = a.student[n * K + lane + 32 * j];
            else a.student[n * K + lane + 32 * j] = 0.0f;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if constexpr (R > 1) {
        if (lane == 0) sh[0][warp] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < R; ++w) m = fmaxf(m, sh[0][w]);
    }
    const float mc = m == -INFINITY ? 0.0f : m * a.c;
    // (a range behind the last column: 0 x 2^-inf)
#pragma unroll
    for (int i = 0; i < HELD; ++i) t += v[i].y * exp2f(fmaf(v[i].x, a.c, -mc));
    for (int i = tid + HELD * 32 * R; i < a.parts; i += 32 * R) {
        const float2 p = row[i];
        t += p.y * exp2f(fmaf(p.x, a.c, -mc));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if constexpr (R > 1) {
        if (lane == 0) sh[1][warp] = t;
        __syncthreads();
        if (warp != 0) return;
        t = 0.0f;
#pragma unroll
        for (int w = 0; w < R; ++w) t += sh[1][w];
    }
    const float lse = __fdiv_rn(m, a.l.tau) + logf(t);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (q[j] != 0.0f) sum += q[j] * (logq[j] - __fdiv_rn(s[j], a.l.tau) + lse);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) { a.lse[n] = lse; a.loss[n] = sum; }
}

// dX from its fp32 sums [splits, N, pitch], four elements a thread; with many ranges (few tokens, hence few elements) four lanes share
// them, each adds every fourth range, and their sums are added in order (N 4, H 576, 64 ranges: 22 us by single threads, 7 by four).
__global__ void __launch_bounds__(256) distill_dx_kernel(const float* src, bf16* __restrict__ dst, int N, int H, int pitch,
                                                         int splits) {
    pdl_begin();
    const int per = H / 4, lanes = splits >= 8 ? 4 : 1, sub = threadIdx.x % lanes, elements = 256 / lanes;
    const size_t n4 = (size_t)N * per, step = (size_t)gridDim.x * elements;
    for (size_t i0 = (size_t)blockIdx.x * elements; i0 < n4; i0 += step) {
        const size_t i = i0 + threadIdx.x / lanes, r = i / per, c = (i - r * per) * 4;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i < n4)
#pragma unroll 8
            for (int s = sub; s < splits; s += lanes) {
                const float4 p = *reinterpret_cast<const float4*>(src + ((size_t)s * N + r) * pitch + c);
                v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
            }
        for (int o = 1; o < lanes; o *= 2) {
            v.x += __shfl_xor_sync(0xffffffffu, v.x, o); v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
            v.z += __shfl_xor_sync(0xffffffffu, v.z, o); v.w += __shfl_xor_sync(0xffffffffu, v.w, o);
        }
        if (sub == 0 && i < n4) *reinterpret_cast<uint2*>(dst + r * H + c) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    }
}

// ------------------------------------------------------------------------------------------ host
template <int KIND, int MODE>
inline mop_status vd_set_smem() {
    return cudaFuncSetAttribute(vd_gemm_kernel<KIND, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                VdTraits<KIND, MODE>::SMEM_BYTES) == cudaSuccess ? MOP_OK : MOP_ERR_CUDA;
}
template <int KIND>
inline mop_status vd_set_smem_rows() {
    mop_status r;
    if ((r = vd_set_smem<KIND, VD_PAIR>()) != MOP_OK) return r;
    if ((r = vd_set_smem<KIND, VD_ONE>()) != MOP_OK) return r;
    return vd_set_smem<KIND, VD_HALF>();
}
inline mop_status vd_init() {
    mop_status r;
    if ((r = vd_set_smem_rows<VD_L>()) != MOP_OK) return r;
    if ((r = vd_set_smem_rows<VD_P>()) != MOP_OK) return r;
    if ((r = vd_set_smem<VD_X, VD_PAIR>()) != MOP_OK) return r;
    if ((r = vd_set_smem<VD_X, VD_ONE>()) != MOP_OK) return r;
    return vd_set_smem<VD_W, VD_PAIR>();
}
template <int KIND, int MODE>
inline mop_status vd_launch(const TcPlan* p, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, VdArgs args, cudaStream_t st) {
    args.stages = VdTraits<KIND, MODE>::stages(args.width);
    const int grid = MODE == VD_PAIR ? p->sm_count & ~1 : p->sm_count;
    return pdl_launch(vd_gemm_kernel<KIND, MODE>, grid, VD_THREADS, VdTraits<KIND, MODE>::SMEM_BYTES, st, a, b, o, args) == cudaSuccess
               ? MOP_OK : MOP_ERR_CUDA;
}
// The mode by the number of rows.
inline int vd_mode(int N) { return N <= 64 ? VD_HALF : N <= 128 ? VD_ONE : VD_PAIR; }
// Rows of a piece of dY in a tile, where it has two; dX's rows are both pieces' then.
inline int vd_piece_rows(int N) { return vd_mode(N) == VD_HALF ? 64 : vd_mode(N) == VD_ONE ? 128 : 0; }
inline int vd_mode_x(int N) { return vd_mode(N) == VD_HALF ? VD_ONE : VD_PAIR; }
inline int vd_row_box(int mode) { return mode == VD_HALF ? 64 : 128; }      // rows of X (or dY) that a CTA copies
template <int KIND>
inline mop_status vd_launch_rows(int mode, const TcPlan* p, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& o, const VdArgs& args,
                                 cudaStream_t st) {
    return mode == VD_PAIR ? vd_launch<KIND, VD_PAIR>(p, a, b, o, args, st)
           : mode == VD_ONE ? vd_launch<KIND, VD_ONE>(p, a, b, o, args, st) : vd_launch<KIND, VD_HALF>(p, a, b, o, args, st);
}
constexpr int VD_SMS = 148;                   // what the rules below count with
// Columns of a tile: the width for which the busiest CTA (or pair) is done first; wide ones where it makes no difference.
// Pairs take one or two chunks of 64 per CTA; with one, X's tile is as much traffic as W's, which counts as 64 columns (N 300, H 2048,
// V 32000 forward: 62 us in 4 rounds of 256 columns, 79 in 7 of 128).  On single CTAs a K block costs about as much whatever the width,
// which counts as 320 columns (forward in us, widths 64, 128, 192 and 256: N 64, H 2048, V 32000 57, 36, 40, 29; N 19, H 3008, V 44608 84,
// 61, 52, 58; N 100, H 2048, V 50304 108, 63, 52, 54; N 16, H 4096, V 64000 138, 104, 99, 88; N 100, H 2048, V 8192, not in L2, 25, 25, 27, 29).
inline int vd_width(int mode, int N, int cols) {
    const bool pair = mode == VD_PAIR;
    const int rows = pair ? (N + 255) / 256 : 1, workers = pair ? VD_SMS / 2 : VD_SMS;
    int pick = 256;
    long long best = 1ll << 60;
    for (int w = 256; w >= 128; w -= pair ? 128 : 64) {
        const long long tiles = (long long)rows * ((cols + w - 1) / w), cost = (tiles + workers - 1) / workers * (w + (pair ? 64 : 320));
        if (cost < best) { best = cost; pick = w; }
    }
    return pick;
}
// [2][rows][pitch] of bf16, the first `cols` columns: 64 of them, `box_rows` rows and `box_pieces` pieces at a time.
inline bool vd_map_pieces(const TcPlan* p, CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows,
                          uint32_t box_pieces) {
    const cuuint64_t dims[3] = {cols, rows, 2};
    const cuuint64_t strides[2] = {pitch * 2, rows * pitch * 2};
    const cuuint32_t box[3] = {64, box_rows, box_pieces};
    const cuuint32_t es[3] = {1, 1, 1};
    return reinterpret_cast<tc_encode_fn>(p->encode)(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
                                                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The same in chunks of 64 columns, two chunks and 64 rows of a piece at a time (an operand whose K are the rows).
inline bool vd_map_pieces_mn(const TcPlan* p, CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch) {
    const cuuint64_t dims[4] = {64, rows, cols / 64, 2};
    const cuuint64_t strides[3] = {pitch * 2, 128, rows * pitch * 2};
    const cuuint32_t box[4] = {64, 64, 2, 1};
    const cuuint32_t es[4] = {1, 1, 1, 1};
    return reinterpret_cast<tc_encode_fn>(p->encode)(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
                                                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// 2-D map over `cols` columns of a bf16 matrix whose rows are `pitch` elements apart, for stores; box = {64 columns, 128 rows}.
inline bool vd_map_out(const TcPlan* p, CUtensorMap* m, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch) {
    return tc_map_2d_pitch(p, m, base, rows, cols, pitch, 128);
}

// Vocabulary columns whose logit gradients are live at a time: as many as keep a piece of dY at 2^28 elements (512 MiB; 1 GiB for the two pieces
// of up to 128 tokens), but at least 8192, which is more than that with more than 32768 tokens; in blocks
// of about equal width.  Wide blocks mean few launches, long sums and few passes over the fp32 sums of dX.  Backward in us, blocks of up to
// 8192, 16384, 32768, 65536 columns and all: N 1537, H 2048, V 50304 930, 829, 770, 722, 723; N 4096, H 7168, V 131072 18150, 17900,
// 17500, 17350, 18500; N 8192 36300, 36550, 37200, 37200, 39500; N 256, H 2048, V 32000 243 in four and 123 in one.
constexpr long long VD_LIVE = 1ll << 28;
inline int vd_block(int N, int V) {
    const long long most = VD_LIVE / N > 8192 ? VD_LIVE / N : 8192;
    const int blocks = (int)((V + most - 1) / most);
    return (int)(((long long)(V + blocks - 1) / blocks + 255) / 256 * 256);
}
// Ranges of K of the dX product, by the makespan of the round-robin in microseconds: a K block of a tile takes 0.3, a unit 2 more, and
// each range its sums' way to L2 and back.
constexpr int VD_MAX_SPLITS = 64;
inline int vd_splits(int N, int H, int width) {
    const bool pair = vd_mode_x(N) == VD_PAIR, pieces = vd_piece_rows(N) > 0;
    const int workers = pair ? VD_SMS / 2 : VD_SMS;
    const int tiles = (pair ? (N + 255) / 256 : 1) * ((H + 255) / 256), kb = (width + 63) / 64;
    const double t_sum = 8e-6 * N * H / 5.0 * (pieces ? 2 : 1);
    int pick = 1;                             // (what is left of a single K block)
    double best = 1e30;
    for (int s = 1; s <= VD_MAX_SPLITS && s <= kb; ++s) {
        if (s == 1 && pieces) continue;                   // (their sums go through memory anyway)
        const double t = ((tiles * (long long)s + workers - 1) / workers) * (((kb + s - 1) / s) * 0.3 + 2.0) + (s > 1 ? t_sum * s : 0.0);
        if (t < 0.97 * best) { best = t; pick = s; }
    }
    return pick;
}

#define DISTILL_BY_K(K, GO)                                       \
    do {                                                          \
        if ((K) <= 32) GO(1);                                     \
        else if ((K) <= 64) GO(2);                                \
        else if ((K) <= 128) GO(4);                               \
        else GO(8);                                               \
    } while (0)

}  // namespace mop
