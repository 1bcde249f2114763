"""The memory that the backward of window attention takes for its sinks, asked on the
host (no GPU needed). Keys that are sinks are worked on in tiles of 128, F of them over
all samples and heads, and each tile in parts with fp32 sums, 128 rows of D for dK and
dV: 1,024 D bytes. Parts are no shorter than an eighth of the launch's work on one
of the P places that the chip has for workgroups (512 at 128 columns, 768 at 64), and the
sinks alone are F tiles' work, so a tile has at most 8 P / F parts, rounded up: all
of them together at most 8 P + F, and one each, which needs no sums, from F = 8 P on."""
import pytest

import paper_2609_23169_amd as ut

PLACES = {64: 512 + 256, 128: 512}


def sums(n, window, sinks, heads, D=128, B=1):
    size = lambda s: ut.ut_swattn_bwd_workspace_size(B, n, n, heads, heads, D, window, s)  # noqa: E731
    assert size(0) > 0
    return size(sinks) - size(0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,window,heads", [(77060, (512, 512), 24), (77060, (128, 128), 24), (40000, (16, 16), 24),
                                            (22879, (2047, 0), 24), (1000000, (512, 512), 24), (9011, (511, 0), 4)])
def test_many_sinks_take_bounded_memory(n, window, heads, D):
    for sinks in (1, 4, 128, 512, 600, 4096, 16384, n // 2, n - 1, n, (1 << 31) - 1):
        tiles = heads * ((min(sinks, n) + 127) // 128)
        got = sums(n, window, sinks, heads, D)
        assert 0 <= got <= (8 * PLACES[D] + tiles) * 1024 * D, (sinks, got)
        if tiles >= 8 * PLACES[D]:
            assert got == 0, sinks


def test_all_keys_as_sinks_need_what_no_window_needs():
    for n, heads in ((77060, 24), (77586, 24)):
        plain = ut.ut_swattn_bwd_workspace_size(1, n, n, heads, heads, 128, (None, None), 0)
        for sinks in (n - 1, n, 1 << 30):
            assert ut.ut_swattn_bwd_workspace_size(1, n, n, heads, heads, 128, (64, 64), sinks) == plain


def test_few_sinks_are_still_cut():
    assert sums(22879, (2047, 0), 4, 24) >= 2 * 24 * 1024 * 128
    assert sums(2048, (127, 0), 4, 3) >= 3 * 3 * 1024 * 128


def test_size_queries_of_many_sinks_are_taken():
    """Parts count as workgroups, which are limited: none of these may be refused for them."""
    for B, n, heads in ((64, 22879, 24), (16, 40000, 64), (1, 1 << 22, 24)):
        for sinks in (4, 4096, n):
            assert ut.ut_swattn_bwd_workspace_size(B, n, n, heads, heads, 128, (16, 0), sinks) > 0
