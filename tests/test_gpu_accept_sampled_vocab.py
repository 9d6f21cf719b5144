"""Sampled acceptance at the largest vocabulary that the call takes: 256 slices of 4096 tokens.  Results are whole numbers and have to be equal."""
import numpy as np
import pytest

from test_gpu_accept_sampled import check, make_case
from test_gpu_parity import pb  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("u_next", [2.0 ** -18, 0.3, 0.9995, 1 - 2.0 ** -22])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("dtype,V", [("f32", 1 << 20), ("bf16", 1 << 20), ("f32", (1 << 20) - 1), ("bf16", (1 << 20) - 1), ("bf16", 526341)])
def test_the_largest_vocabularies(pb, dtype, V, drawn, u_next):
    """The token lies in the first slice, in the middle and in the last ones."""
    x = make_case(np.random.default_rng(V % 1000 + drawn), dtype, 1, 3, V, drawn, sharp=2.0, sizes=[3])
    x["u"][:] = 0.9  # (hardly anything passes)
    x["u_next"][:] = u_next
    want = check(pb, x)
    slices = (V + 4095) // 4096
    if not drawn or not 0.1 < u_next < 0.9999:
        assert abs(int(want[2][0]) / 4096 - u_next * slices) < 4 + 0.05 * slices
