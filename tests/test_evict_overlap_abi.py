"""An eviction's outputs may overlap neither its inputs nor each other: the selection
writes kept_idx and len_out while other workgroups still read weights and lengths,
and the move reads kept_idx while it writes the rest. On the host, before any
launch (no GPU needed)."""
import ctypes

import pytest

import paper_2609_23169_amd as ut
from test_swattn_cache_abi import BAD, _ev

B, CAP, CAPO, HK, D, KEEP = 2, 300, 100, 2, 64, 100
ROW = HK * D * 2
SIZES = {"k": B * CAP * ROW, "v": B * CAP * ROW, "w": B * HK * CAP * 4, "lens": B * 4, "ko": B * CAPO * ROW,
         "vo": B * CAPO * ROW, "wo": B * HK * CAPO * 4, "lo": B * 4, "idx": B * HK * KEEP * 4}
NAMES = {"k": "k_cache", "v": "v_cache", "w": "weights", "lens": "cache_len", "ko": "k_out", "vo": "v_out",
         "wo": "weights_out", "lo": "len_out", "idx": "kept_idx"}
AT = {x: 0x10000000 * (i + 1) for i, x in enumerate(SIZES)}
at = ctypes.c_void_p


def refused(**kw):
    assert _ev(**kw) == BAD
    return ut.last_error()


@pytest.mark.parametrize("out", ["ko", "vo", "wo", "lo", "idx"])
@pytest.mark.parametrize("other", list(SIZES))
def test_outputs_lie_apart_from_all_others(out, other):
    if out == other:
        return
    step = 16 if {out, other} & {"k", "v", "ko", "vo"} else 4
    for place in (AT[other], AT[other] + (SIZES[other] - step) // step * step, AT[other] - SIZES[out] + step):
        text = refused(**{out: at(place)})
        assert f"{NAMES[out]} overlaps {NAMES[other]}" in text or f"{NAMES[other]} overlaps {NAMES[out]}" in text, text


def test_interleaved_outputs_of_one_buffer_are_taken():
    """As far as the next check, that of the lengths."""
    k = AT["ko"]
    wide = (HK * D, HK * D, 3 * HK * D, 3 * HK * D)
    for by in (ROW, 2 * ROW, -ROW, -2 * ROW, 5 * ROW):
        assert _ev(ko=at(k), vo=at(k + by), strides=wide, lens=None) == BAD
        assert "cache_len is NULL" in ut.last_error()
    for by in (0, 16, ROW - 16, 2 * ROW + 16, -16, 3 * ROW):
        assert "v_out overlaps k_out" in refused(ko=at(k), vo=at(k + by), strides=wide)
    # other strides than each other's
    assert "v_out overlaps k_out" in refused(ko=at(k), vo=at(k + ROW), strides=wide[:3] + (4 * HK * D,))
