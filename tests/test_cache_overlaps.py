"""What the binding refuses before any call is made, by its own checks on host tensors (no GPU needed)."""
import math

import pytest
import torch

from test_abi import pb  # noqa: F401
from test_cache_refusals import INVALID, UNSUPPORTED, WORKSPACE, attention, observe, rule_of


def test_workspaces_of_another_device_or_with_gaps_are_refused(pb):
    cpu, meta = torch.device("cpu"), torch.device("meta")
    ws = torch.empty(512, dtype=torch.uint8)
    assert pb._workspace(512, cpu, ws) is ws
    with pytest.raises(TypeError):
        pb._workspace(256, meta, ws)
    for gaps in (torch.empty(1, dtype=torch.uint8).expand(512), torch.empty(1024, dtype=torch.uint8)[::2], torch.empty(32, 32, dtype=torch.uint8).t()):
        with pytest.raises(TypeError):
            pb._workspace(256, cpu, gaps)
    with pytest.raises(ValueError):
        pb._workspace(513, cpu, ws)


def test_overlaps(pb):
    base = torch.zeros(64)
    pb._apart(base[:10], "out", None, base[10:20], torch.zeros(3))
    pb._apart(base[5:5], "out", base)  # nothing to overlap
    pb._apart(None, "out", base)
    for other in (base, base[9:10], base.view(torch.int32)[:1]):
        with pytest.raises(ValueError, match="out: overlaps"):
            pb._apart(base[:10], "out", torch.zeros(1), other)
    pb._same_or_apart(base[:10], base[:10], "out")
    with pytest.raises(ValueError):
        pb._same_or_apart(base[1:11], base[:10], "out")


def test_workspace_of_the_attention_holds_what_plans_use(pb):
    """At most 1024 partial results of 66 KB, 512 where there are few units, and no more than there are stages."""
    piece = 66 << 10
    for args, most in (((1, 1, 1, 128, 0), 1), ((1, 1, 32, 128, 1024), 512), ((2, 128, 50, 64, 1 << 20), 512), ((32, 64, 32, 128, 4096), 1024), ((1, 128, 1, 64, 60), 6)):
        got = pb.workspace_bytes(pb.WS_GROUPED_ATTENTION, *args)
        assert most * piece <= got <= most * piece + 16 * args[0] * args[2] + 1024, args


def test_scales_and_paths_beyond_all_use_are_refused(pb):
    for scale in (math.nextafter(2.0 ** 64, math.inf) * 1.001, 1e38, 3e38):
        assert attention(pb, rule=rule_of(pb, scale)) == INVALID and observe(pb, rule=rule_of(pb, scale)) == INVALID
    for scale in (2.0 ** 64, 2.0 ** -140):  # what is refused then is the workspace
        assert attention(pb, rule=rule_of(pb, scale), ws=None) == WORKSPACE
    assert observe(pb, stride=65537) == UNSUPPORTED and observe(pb, stride=1 << 24, H=2) == UNSUPPORTED
