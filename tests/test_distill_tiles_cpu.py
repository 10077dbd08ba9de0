"""Host-side rules of the distillation's tiles (no device here)."""
from test_gpu_distill_tiles import TILES
from test_host_rules_cpu import run_host_program


def test_the_tile_shapes_that_the_device_tests_mean_to_reach(tmp_path):
    """The widths that the rule picks for them, and the rounds of the SMs that the tiles make: a change of the rule must not drop one."""
    assert {(w, r > 1) for w, r in TILES.values()} >= {(128, True), (192, False), (192, True), (256, True)}
    cases = "".join(f"{{{N}, {V}, {w}, {r}}}, " for (N, _, V, _), (w, r) in TILES.items())
    run_host_program(tmp_path, r"""
#include "distill.cuh"
#include <cstdio>
using namespace mop;
int main() {
    int bad = 0;
    const int cases[][4] = {""" + cases + r"""};
    for (const auto& c : cases) {
        const int mode = vd_mode(c[0]), w = vd_width(mode, c[0], c[1]), workers = mode == VD_PAIR ? VD_SMS / 2 : VD_SMS;
        const int tiles = (mode == VD_PAIR ? ceil_div(c[0], 256) : 1) * ceil_div(c[1], w), rounds = ceil_div(tiles, workers);
        if (w != c[2] || rounds != c[3]) { std::printf("N %d V %d: %d columns, %d rounds\n", c[0], c[1], w, rounds); ++bad; }
    }
    return bad;
}
""")


def test_bytes_of_the_logit_gradients():
    """One block of columns: 2^28 elements of each piece, so twice the bytes up to 128 tokens; with many tokens no fewer than 8192 columns."""
    import __graft_entry__
    __graft_entry__.build()
    from paper_2607_01844_b200 import binding
    need = binding.lib().mop_vocab_distill_bwd_workspace_bytes
    H, K = 8, 1
    for N, V, columns, pieces in ((64, 1 << 24, 1 << 22, 2), (128, 1 << 24, 1 << 21, 2), (129, 1 << 24, None, 1), (32768, 1 << 20, 8192, 1),
                                  (100000, 1 << 20, 8192, 1)):
        columns = columns or (1 << 28) // N // 256 * 256
        dY = 2 * pieces * N * columns
        # beside it: sorted entries, 2 bytes per token and 64 columns of the whole vocabulary, fp32 sums of dX in up to 64 ranges
        rest = N * K * 8 + N * (V // 64 + 1) * 2 + 64 * pieces * N * 32 * 4 + N * 8 + 4096
        assert dY * 0.99 <= need(N, H, V, K) <= dY + rest
