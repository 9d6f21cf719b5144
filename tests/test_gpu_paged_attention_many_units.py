"""Attention over a paged cache on both sides of the number of units from which none is cut, in every shape of the waves."""
import numpy as np
import pytest

from cache_util import f64, make_inputs, rule_of
from paged_util import codes_of, numbers
from oracle import paged_cache as ref
from paper_2402_13485_amd import synth
from test_gpu_paged_attention import check_attention, run_attention
from test_gpu_parity import pb  # noqa: F401

pytestmark = pytest.mark.gpu


def shared_pool_case(rng, dtype, codes, B, Hk, d, lens, T_max, n_pages=48, R=16):
    """Many sequences over few pages, any page in any place of their tables; trees of one or two nodes but for the first sequences."""
    shapes = [synth.chain_tree(T_max if b < 2 else 1 + b % min(2, T_max)) for b in range(B)]
    x = make_inputs(rng, dtype, Hk, Hk, d, shapes, [0] * B, T_max=T_max)
    x.update(R=R, seq_lens=np.array(lens, np.int32), page_table=rng.integers(0, n_pages, (B, -(-max(lens) // R))).astype(np.int32))
    for name in "kv":
        shape = (n_pages, Hk, R, d)
        x[name + "_pages"] = codes_of(rng, *shape) if codes else numbers(rng, dtype, *shape)
        x[name + "_scale"] = rng.integers(118, 122, shape[:3]).astype(np.uint8) if codes else None
        x[name + "64"] = ref.decode(x[name + "_pages"], x[name + "_scale"]) if codes else f64(x[name + "_pages"])
    return x


@pytest.mark.parametrize("T_max,dtype,codes", [(1, "bf16", True), (1, "f32", False), (20, "bf16", False), (20, "f32", True), (70, "bf16", True), (70, "f32", False)])
@pytest.mark.parametrize("B", [255, 256, 257])
def test_units_around_the_most_that_are_cut(pb, B, T_max, dtype, codes):
    """4080 units, of which the last round's and those of long sequences are cut, 4096 and 4112, none of which is; ragged, two long sequences among short
    ones, one empty, batches of several times 64 sequences."""
    rng = np.random.default_rng(B + T_max)
    lens = [int(n) for n in rng.integers(1, 120, B)]
    lens[1], lens[B - 2], lens[5] = 900, 640, 0
    x = shared_pool_case(rng, dtype, codes, B, 16, 64, lens, T_max)
    check_attention(x, rule_of(64), *run_attention(pb, x, rule_of(64)))
