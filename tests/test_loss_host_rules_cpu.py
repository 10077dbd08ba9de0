"""Host-side rules of the auxiliary losses' kernels, compiled and run without a device."""
from test_host_rules_cpu import run_host_program


def test_every_token_block_of_every_tile_belongs_to_one_range(tmp_path):
    """The dW_r product's ranges: each token block of each tile is taken once, a cut tile's sums lie in slots of their own, and the
    summing kernel looks for them where they were left."""
    run_host_program(tmp_path, r"""
#include "balance.cuh"
#include <cstdio>
#include <map>
#include <vector>
using namespace mop;
int main() {
    int cuts = 0;
    const int Ts[] = {1, 64, 65, 200, 1537, 4096, 16384, 20000}, ds[] = {8, 256, 264, 1000, 2048, 7168}, Es[] = {1, 8, 64, 128, 129, 200, 256, 300, 384, 512, 1000, 1024};
    for (int T : Ts) for (int d : ds) for (int E : Es) {
        const BalCut c = bal_cut(T, d, E);
        const int total = c.total(), pairs = (total + c.range - 1) / c.range;
        std::map<std::pair<int, int>, int> taken;
        std::map<std::pair<int, int>, int> slots;
        for (int p = 0; p < pairs; ++p)
            for (int u = p * c.range, end = u + c.range < total ? u + c.range : total, to; u < end; u = to) {
                const int tile = c.tile_at(u);
                to = c.start(tile) + c.cost(tile);
                if (to > end) to = end;
                for (int kb = c.block_at(tile, u); kb < c.block_at(tile, to); ++kb) ++taken[{tile, kb}];
                if (p < c.first_pair(tile) || p > c.last_pair(tile)) { std::printf("range %d of tile %d\n", p, tile); return 1; }
                if (c.first_pair(tile) != c.last_pair(tile) && slots[{p, c.first_pair(tile) < p ? 0 : 1}]++) { std::printf("slot twice\n"); return 1; }
            }
        for (int tile = 0; tile < c.tiles(); ++tile)
            for (int p = c.first_pair(tile); p <= c.last_pair(tile); ++p)
                if (c.first_pair(tile) != c.last_pair(tile) && !slots.count({p, p == c.first_pair(tile) ? 1 : 0})) { std::printf("missing sums\n"); return 1; }
        if (pairs > BAL_PAIRS || (int)taken.size() != c.tiles() * c.kb || c.tiles() != ((d + 255) / 256) * ((E + 255) / 256)) {
            std::printf("T %d d %d E %d: %d pairs, %d of %d blocks\n", T, d, E, pairs, (int)taken.size(), c.tiles() * c.kb);
            return 1;
        }
        for (auto& t : taken) if (t.second != 1) return 1;
        cuts += bal_is_cut(c);
    }
    return cuts < 50;
}
""")


def test_column_blocks_cover_the_vocabulary_in_whole_tiles(tmp_path):
    """Blocks of the logit gradients: whole tiles (256 columns), at most 2^28 elements or 8192 columns, none of them empty, and the
    ranges of the dX product never more than the widest block's K blocks."""
    run_host_program(tmp_path, r"""
#include "distill.cuh"
#include <cstdio>
using namespace mop;
int main() {
    const int Ns[] = {1, 64, 1537, 2304, 4096, 8192, 8200, 65536, 1 << 20}, Vs[] = {8, 64, 4096, 8192, 8200, 32000, 50304, 131072, 1 << 20}, Hs[] = {8, 512, 2040, 7168};
    for (int N : Ns) for (int V : Vs) {
        const int vc = vd_block(N, V), blocks = (V + vc - 1) / vc;
        const long long most = VD_LIVE / N > 8192 ? VD_LIVE / N : 8192;
        if (vc < 1 || vc % 256 || vc > most + 255 || (blocks - 1) * (long long)vc >= V) { std::printf("N %d V %d: %d\n", N, V, vc); return 1; }
        for (int H : Hs) {
            const int width = V < vc ? V : vc, s = vd_splits(N, H, width);
            if (N == 2304 && V == 4096 && H == 2040 && (s != 1 || blocks != 1)) return 1;      // the case that stores dX at once
            if (s < 1 || s > VD_MAX_SPLITS || s > (width + 63) / 64) return 1;
        }
    }
    return 0;
}
""")


def test_workspace_sizes_need_no_device_and_take_every_shape():
    import ctypes

    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_01844_b200 import binding
    lib = binding.lib()
    for T in (0, 1, 63, 5000):
        for E, k in ((1, 1), (8, 2), (200, 8), (1024, 32)):
            for path in (binding.GEMM_AUTO, binding.GEMM_SCALAR):
                shape = binding.MopShape(T, 264, E, k, 64, 0, 0, 0, 0, path, 0, 0)
                sizes = [lib.mop_moe_balance_workspace_bytes(ctypes.byref(shape), 3, b) for b in (0, 1)]
                assert all(s % 256 == 0 for s in sizes) and (T == 0 or min(sizes) > 0)
    assert lib.mop_moe_balance_workspace_bytes(ctypes.byref(binding.MopShape(8, 252, 8, 2, 64, 0, 0, 0, 0, 0, 0, 0)), 1, 1) == 0
    for n in (0, -1, 1 << 28):
        assert lib.mop_moe_balance_workspace_bytes(ctypes.byref(binding.MopShape(8, 256, 8, 2, 64, 0, 0, 0, 0, 0, 0, 0)), n, 1) == 0
    for N in (0, 1, 300, 1 << 20):
        assert lib.mop_vocab_distill_workspace_bytes(N, 72, 1000, 256) >= 256 and lib.mop_vocab_distill_bwd_workspace_bytes(N, 72, 1000, 1) >= 256
    for bad in ((-1, 64, 64, 1), (1, 60, 64, 1), (1, 64, 60, 1), (1, 64, 64, 0), (1, 64, 64, 257), (1 << 30, 64, 64, 1), (1, 8, (1 << 30) + 8, 1),
                (1 << 29, 64, 1 << 20, 1), (1 << 29, 1 << 14, 64, 1)):
        assert lib.mop_vocab_distill_workspace_bytes(*bad) == 0 and lib.mop_vocab_distill_bwd_workspace_bytes(*bad) == 0
    assert lib.mop_moe_balance_loss_fwd(None, 1, *[None] * 9) == 1
    assert lib.mop_moe_balance_loss_bwd(None, 1, *[None] * 7, 0, *[None] * 6) == 1
    f = ctypes.c_float
    for tau, code in ((0.0, 1), (-2.0, 1), (float("nan"), 1), (float("inf"), 1), (1.0, 1)):
        assert lib.mop_vocab_distill_fwd(0, 4, 64, 64, 2, *[None] * 5, f(tau), *[None] * 5) == code
    assert lib.mop_vocab_distill_fwd(0, 4, 60, 64, 2, *[None] * 5, f(1.0), *[None] * 5) == 3
    assert lib.mop_vocab_distill_bwd(0, 4, 64, 64, 257, *[None] * 5, f(1.0), *[None] * 7) == 2
    assert lib.mop_vocab_distill_bwd(99, 4, 64, 64, 2, *[None] * 5, f(1.0), *[None] * 7) == 1


def test_tiles_stages_and_boxes_fit_shared_memory(tmp_path):
    """Every kind in every mode: the ring, the store boxes and the barriers fit 227 KiB, a stage is whole swizzle atoms, a half-height
    operand is followed by enough of its own stage for the 128 rows that the instruction reads; every width that the rule picks covers the
    columns, and its entries and partial sums are counted in the same units everywhere."""
    run_host_program(tmp_path, r"""
#include "distill.cuh"
#include <cstdio>
using namespace mop;
template <int KIND, int MODE> int check() {
    using Tr = VdTraits<KIND, MODE>;
    int bad = Tr::SMEM_BYTES > 232448;
    for (int w = Tr::PAIR ? 128 : 64; w <= 256; w += Tr::PAIR ? 128 : 64) {
        const int st = Tr::stages(w), bytes = Tr::PAIR ? T2_STAGE_BYTES : Tr::A_BYTES + w * TC_BK * 2;
        bad += st < 3 || st > Tr::STAGES || st * bytes > Tr::RING_BYTES || bytes % 1024 || bytes < T2_A_BYTES;
        bad += (2 * Tr::STAGES + 4) * 8 + 8 > TC_BAR_BYTES;
    }
    if (bad) std::printf("kind %d mode %d: %d bytes\n", KIND, MODE, Tr::SMEM_BYTES);
    return bad;
}
int main() {
    int bad = check<VD_L, VD_PAIR>() + check<VD_L, VD_ONE>() + check<VD_L, VD_HALF>() + check<VD_P, VD_PAIR>() + check<VD_P, VD_ONE>() +
              check<VD_P, VD_HALF>() + check<VD_X, VD_PAIR>() + check<VD_X, VD_ONE>() + check<VD_X, VD_HALF>() + check<VD_W, VD_PAIR>() + check<VD_R, VD_PAIR>();
    bool seen[5] = {};
    for (int N : {1, 64, 65, 128, 129, 256, 257, 8192})
        for (int V = 8; V < 200000; V += V < 1000 ? 8 : 1000) {
            const int mode = vd_mode(N), w = vd_width(mode, N, V);
            if (w < 128 || w > 256 || w % (mode == VD_PAIR ? 128 : 64)) { std::printf("N %d V %d: %d\n", N, V, w); ++bad; }
            else if (mode != VD_PAIR) seen[w / 64] = true;
            if (mode == VD_HALF ? N > 64 : mode == VD_ONE ? N > 128 : N <= 128) ++bad;
        }
    return bad || !(seen[2] && seen[3] && seen[4]);
}
""")
