"""Cache calls whose launches would reach 2^32 threads - caches of a few slots with
millions of sample-heads - are refused before any launch, and their size query
returns 0. On the host (no GPU needed; pointers are never used on these paths)."""
import ctypes

import pytest

import paper_2609_23169_amd as ut
from test_swattn_cache_abi import BAD, FAKE, _ca, _ev


@pytest.mark.parametrize("B,cap,Hq,Hk,D", [(1 << 24, 1, 1, 1, 64), (1 << 23, 4, 2, 2, 64), (1 << 19, 3, 64, 32, 8)])
def test_scores_of_few_rows(B, cap, Hq, Hk, D):
    """A workgroup 256 slots of a key head behind the attention, where that is a launch of its own."""
    size = dict(B=B, T=1, cap=cap, Hq=Hq, Hk=Hk, D=D)
    assert _ca(**size, wout=FAKE) == BAD and "too large" in ut.last_error()
    assert ut.ut_cache_attn_workspace_size(B, 1, cap, Hq, Hk, D, with_weights=True) == 0


def test_weights_alone():
    size = dict(B=1 << 20, T=2, cap=5, Hq=8, Hk=8, D=64, wout=FAKE)
    assert _ca("weights", **size) == BAD and "too large" in ut.last_error()
    assert _ca("weights", **dict(size, B=(1 << 20) - 1, lens=None)) == BAD and "cache_len is NULL" in ut.last_error()


def test_eviction():
    p = lambda i: ctypes.c_void_p(i << 44)  # noqa: E731
    far = dict(zip(("k", "v", "w", "lens", "ko", "vo", "wo", "lo", "idx"), map(p, range(1, 10))))
    size = dict(B=1 << 15, Hk=1 << 9, cap=7, capo=3, keep=3, sinks=1, recent=1, D=8)
    assert _ev(**far, **size) == BAD and "too large" in ut.last_error()
    assert _ev(**dict(far, lens=None), **dict(size, B=(1 << 15) - 1)) == BAD and "cache_len is NULL" in ut.last_error()
