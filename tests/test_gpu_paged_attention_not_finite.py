"""Rows that are not finite in attention over a paged cache, where scores differ by more than fp32 weights can: a softmax gives every row that a
query sees a weight above zero, so an infinity or a NaN reaches the query's result wherever the row lies, in whatever order the rows
come, and however the rows are cut into ranges.  Against the float64 definition of oracle/paged_cache.py."""
import numpy as np
import pytest

from cache_util import f64, rule_of
from oracle import paged_cache as ref
from paged_util import make_case
from paper_2402_13485_amd import synth
from test_gpu_paged_attention import check_attention, run_attention
from test_gpu_parity import pb  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]


def set_rows(x, value_of):
    """K of row j of the first sequence: value_of[j] throughout"""
    for value in np.unique(value_of):
        rows = np.flatnonzero(value_of == value)
        page, at = x["page_table"][0, rows // x["R"]], rows % x["R"]
        values = np.full(x["k64"].shape[3], value, np.float32)
        if x["k_scale"] is not None:
            codes, scale = ref.quantise(values)
            x["k_pages"][page, :, at], x["k_scale"][page, :, at] = codes, scale
            x["k64"][page, :, at] = ref.decode(codes[None], [scale])[0]
        else:
            x["k_pages"][page, :, at] = synth.from_float(values, x["dtype"])
            x["k64"][page, :, at] = f64(synth.from_float(values, x["dtype"]))


def set_value(x, j, column, value):
    """An entry of V of row j of the first sequence and head"""
    page, at = x["page_table"][0, j // x["R"]], j % x["R"]
    if x["v_scale"] is not None:
        x["v_pages"][page, 0, at, column] = 0x7f
        value = np.nan
    else:
        x["v_pages"][page, 0, at, column] = synth.from_float(np.array([value], np.float32), x["dtype"])[0]
    x["v64"][page, 0, at, column] = value


@pytest.mark.parametrize("order", ["rising", "falling"])
@pytest.mark.parametrize("L", [60, 200, 4000])
@pytest.mark.parametrize("T", [1, 9, 20, 70])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_infinities_of_rows_that_weigh_next_to_nothing(pb, dtype, codes, T, L, order):
    """Scores over a range of 288 (a weight of 1e-125: zero in fp32), that rise or fall with the rows; infinities of both signs and a NaN in rows at
    both ends and in the middle, alone in a column and together.  One range, and several that are joined."""
    rng = np.random.default_rng(L + T)
    x = make_case(rng, dtype, codes, 2, 1, 64, [synth.chain_tree(T)], [L], 16)
    steps = np.arange(L) * 24 // L
    set_rows(x, 12.0 * (steps if order == "rising" else steps[::-1]) / 24)
    x["q"][...] = synth.from_float(np.full(x["q"].shape, 3.0, np.float32), dtype)
    for j, column, value in ((0, 3, np.inf), (L - 1, 5, -np.inf), (L // 2, 9, np.nan), (1, 17, -np.inf), (L - 2, 17, np.inf), (L // 3, 40, np.inf), (2, 40, np.inf)):
        set_value(x, j, column, value)
    out, lse = run_attention(pb, x, rule_of(64))
    got = synth.as_float(out[0]).astype(np.float64)
    for column in (9, 17):
        assert np.isnan(got[..., column]).all()
    check_attention(x, rule_of(64), out, lse)


@pytest.mark.parametrize("where", ["own row", "last row", "second half"])
@pytest.mark.parametrize("T,L", [(1, 33), (1, 200), (1, 5000), (9, 65), (20, 4000), (70, 4000)])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_scores_that_are_no_numbers(pb, dtype, codes, T, L, where):
    """NaN in K of rows that a query sees: its results are NaN, also where a range of rows or a wave has nothing but such rows."""
    rng = np.random.default_rng(L + T)
    x = make_case(rng, dtype, codes, 4, 2, 64, [synth.chain_tree(T), synth.chain_tree(T)], [L, L], 16)
    clean = run_attention(pb, x, rule_of(64))
    if where == "own row":  # of the first node, which all others see
        x["k_tree"][0, :, 0, 7] = synth.from_float(np.array([np.nan], np.float32), dtype)[0]
    for j in {"own row": [], "last row": [L - 1], "second half": range(L // 2, L)}[where]:
        page, at = x["page_table"][0, j // 16], j % 16
        x["k_pages"][page, :, at, 7] = 0x7f if codes else synth.from_float(np.array([np.nan], np.float32), dtype)[0]
    out, lse = run_attention(pb, x, rule_of(64))
    assert np.isnan(synth.as_float(out[0])).all() and np.isnan(lse[0]).all()
    assert (out[1].view(np.uint8) == clean[0][1].view(np.uint8)).all() and (lse[1] == clean[1][1]).all()
