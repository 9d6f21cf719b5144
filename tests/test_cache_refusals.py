"""What the calls of a bounded cache refuse, on the host, before anything is enqueued (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from test_abi import pb  # noqa: F401

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
OK = 0x1000  # never dereferenced: validation fails first
ODD = 0x1004


def rule_of(pb, scale=0.1, cap=0.0, window=0):
    return ctypes.byref(pb._ScoreRule(scale, cap, window, None))


def attention(pb, dt=None, H=8, H_kv=2, d=128, rule=None, tree=None, L_max=64, ws=OK, ws_bytes=1 << 40, **ptr):
    a = dict(q=OK, k=OK, v=OK, kt=OK, vt=OK, lens=OK, position=None, dropped=None, out=OK)
    a.update(ptr)
    tree = tree or pb._Tree(2, 16, OK, OK, OK, OK, OK)
    return pb.load_library().propd_grouped_attention(ctypes.byref(tree), pb.PROPD_BF16 if dt is None else dt, H, H_kv, d, rule or rule_of(pb), a["q"], a["k"], a["v"],
                                                     a["kt"], a["vt"], a["lens"], a["position"], a["dropped"], L_max, a["out"], None, ws, ws_bytes, None)


def test_attention_refusals(pb):
    for dt in (pb.PROPD_BF16, pb.PROPD_F32):
        assert attention(pb, dt, ws=None) == WORKSPACE and attention(pb, dt, ws_bytes=100) == WORKSPACE
        assert attention(pb, dt, d=96) == UNSUPPORTED and attention(pb, dt, d=256) == UNSUPPORTED
        assert attention(pb, dt, H=8, H_kv=3) == INVALID and attention(pb, dt, H=0) == INVALID and attention(pb, dt, H_kv=0) == INVALID
        for name in ("q", "k", "v", "kt", "vt", "out"):
            assert attention(pb, dt, **{name: ODD}) == INVALID and attention(pb, dt, **{name: None}) == INVALID, name
        assert attention(pb, dt, ws=ODD) == INVALID and attention(pb, dt, lens=None) == INVALID and attention(pb, dt, L_max=-1) == INVALID
        assert attention(pb, dt, tree=pb._Tree(2, 129, OK, OK, OK, OK, OK)) == INVALID
        assert attention(pb, dt, tree=pb._Tree(0, 16, OK, OK, OK, OK, OK)) == INVALID
        assert attention(pb, dt, tree=pb._Tree(2, 16, OK, OK, OK, OK, None)) == INVALID
        assert attention(pb, dt, tree=pb._Tree(2, 16, OK, OK, OK, OK, 0x1008)) == INVALID
        assert attention(pb, dt, L_max=(1 << 30) + 1) == UNSUPPORTED
        assert attention(pb, dt, tree=pb._Tree((1 << 20) + 1, 128, OK, OK, OK, OK, OK)) == UNSUPPORTED
    assert attention(pb, 2) == INVALID
    # no cache rows: K and V of the cache may be missing (what is refused then is the workspace)
    assert attention(pb, L_max=0, k=None, v=None, ws=None) == WORKSPACE


@pytest.mark.parametrize("scale,cap,window", [(0.0, 0.0, 0), (-1.0, 0.0, 0), (math.nan, 0.0, 0), (math.inf, 0.0, 0), (1.0, -1.0, 0), (1.0, math.nan, 0),
                                              (1.0, math.inf, 0), (1.0, 2e3, 0), (1.0, 1e-4, 0), (1.0, 0.0, -1), (1.0, 0.0, (1 << 24) + 1)])
def test_rules_that_are_refused(pb, scale, cap, window):
    assert attention(pb, rule=rule_of(pb, scale, cap, window)) == INVALID
    assert observe(pb, rule=rule_of(pb, scale, cap, window)) == INVALID


def observe(pb, dt=None, H=8, H_kv=2, d=128, rule=None, decay=0.5, stride=8, L_max=64, tree=None, **ptr):
    a = dict(len=OK, path=OK, q=OK, lse=OK, k=OK, kt=OK, lens=OK, position=OK, weight=OK, position_out=OK, weight_out=OK)
    a.update(ptr)
    tree = tree or pb._Tree(2, 16, OK, OK, OK, OK, OK)
    return pb.load_library().propd_cache_observe(ctypes.byref(tree), pb.PROPD_BF16 if dt is None else dt, H, H_kv, d, rule or rule_of(pb), decay, a["len"], a["path"],
                                                 stride, a["q"], a["lse"], a["k"], a["kt"], a["lens"], None, a["position"], a["weight"], L_max,
                                                 a["position_out"], a["weight_out"], None)


def test_observe_refusals(pb):
    assert observe(pb, 9) == INVALID and observe(pb, d=80) == UNSUPPORTED and observe(pb, H=9) == INVALID
    assert observe(pb, L_max=0) == INVALID and observe(pb, stride=0) == INVALID
    for decay in (0.0, -0.5, 1.5, math.nan):
        assert observe(pb, decay=decay) == INVALID
    for name in ("len", "path", "q", "lse", "k", "kt", "lens", "weight", "weight_out", "position", "position_out"):
        assert observe(pb, **{name: None}) == INVALID, name  # position and position_out: one without the other
    for name in ("q", "k", "kt"):
        assert observe(pb, **{name: ODD}) == INVALID
    assert observe(pb, tree=pb._Tree(1 << 24, 16, OK, OK, OK, OK, OK)) == UNSUPPORTED
    assert observe(pb, L_max=(1 << 30) + 1) == UNSUPPORTED
    assert observe(pb, stride=(1 << 30) - 1) == UNSUPPORTED


def evict(pb, dt=None, B=2, H_kv=2, d=128, L_max=64, budget=16, recent=4, sinks=0, k=OK, v=OK, rows=(OK,) * 4, out=(OK,) * 4, ws=OK, ws_bytes=1 << 40):
    r, o = pb._CacheRows(*rows), pb._CacheRows(*out)
    return pb.load_library().propd_cache_evict(B, pb.PROPD_BF16 if dt is None else dt, H_kv, d, L_max, budget, recent, sinks, k, v, ctypes.byref(r), ctypes.byref(o),
                                               ws, ws_bytes, None)


def test_evict_refusals(pb):
    assert evict(pb, 5) == INVALID and evict(pb, B=0) == INVALID and evict(pb, H_kv=0) == INVALID and evict(pb, L_max=0) == INVALID
    assert evict(pb, budget=0) == INVALID and evict(pb, budget=65) == INVALID and evict(pb, recent=-1) == INVALID and evict(pb, sinks=-1) == INVALID
    assert evict(pb, k=None) == INVALID and evict(pb, v=ODD) == INVALID and evict(pb, ws=ODD) == INVALID
    assert evict(pb, ws=None) == WORKSPACE and evict(pb, ws_bytes=64) == WORKSPACE
    assert evict(pb, d=12) == UNSUPPORTED and evict(pb, d=1 << 24) == UNSUPPORTED and evict(pb, B=1 << 20) == UNSUPPORTED
    for i in range(4):
        some = tuple(None if j == i else OK for j in range(4))
        assert evict(pb, rows=some) == INVALID and evict(pb, out=some) == INVALID


def rotary(pb, dt=None, B=2, S=8, H=4, H_kv=2, d=128, rot=64, n_axes=1, offset_axes=1, **ptr):
    a = dict(inv=OK, offset=OK, q=OK, k=OK, q_out=OK, k_out=OK)
    a.update(ptr)
    return pb.load_library().propd_rotary(pb.PROPD_BF16 if dt is None else dt, B, S, H, H_kv, d, rot, 0, n_axes, None, a["inv"], None, a["offset"], offset_axes, None,
                                          a["q"], a["k"], a["q_out"], a["k_out"], None)


def test_rotary_refusals(pb):
    assert rotary(pb, 7) == INVALID and rotary(pb, B=0) == INVALID and rotary(pb, S=0) == INVALID and rotary(pb, H=0) == INVALID and rotary(pb, H_kv=-1) == INVALID
    assert rotary(pb, rot=256) == INVALID and rotary(pb, rot=0) == INVALID and rotary(pb, rot=24) == UNSUPPORTED and rotary(pb, d=100) == UNSUPPORTED
    assert rotary(pb, n_axes=0) == INVALID and rotary(pb, n_axes=3, offset_axes=2) == INVALID and rotary(pb, offset_axes=3) == INVALID
    for name in ("inv", "offset", "q", "k", "q_out", "k_out"):
        assert rotary(pb, **{name: None}) == INVALID, name
    for name in ("q", "k", "q_out", "k_out"):
        assert rotary(pb, **{name: ODD}) == INVALID, name
    assert rotary(pb, H=65535) == UNSUPPORTED and rotary(pb, B=1 << 20, S=1 << 20) == UNSUPPORTED


def test_workspace_sizes(pb):
    assert pb.workspace_bytes(pb.WS_GROUPED_ATTENTION, 1, 1, 1, 128, 0) > 0
    assert pb.workspace_bytes(pb.WS_GROUPED_ATTENTION, 16, 128, 40, 128, 4096) < 160 << 20  # partial results of the ranges, bounded
    assert pb.workspace_bytes(pb.WS_GROUPED_ATTENTION, 16, 129, 40, 128, 4096) == 0
    assert pb.workspace_bytes(pb.WS_CACHE_EVICT, 2, 0, 8, 0, 4096) >= 2 * 8 * 4096 * 4
    assert pb.workspace_bytes(pb.WS_CACHE_EVICT, 2, 0, 0, 0, 4096) == 0


def test_tensors_in_host_memory_are_refused(pb):
    z = torch.zeros
    i32 = dict(dtype=torch.int32)
    tree = pb.Tree(z(1, **i32), z(1, 4, **i32), z(1, 4, **i32), z(1, 4, **i32), z(1, 4, 2, dtype=torch.int64))
    rows = pb.CacheRows(z(1, **i32), z(1, **i32), z(1, 2, 8, **i32), z(1, 2, 8))
    q, k, kt = z(1, 4, 4, 64), z(1, 2, 8, 64), z(1, 2, 4, 64)
    with pytest.raises(TypeError):
        pb.propd_grouped_attention(tree, q, k, k.clone(), kt, kt.clone(), rows.seq_lens, 0.1)
    with pytest.raises(TypeError):
        pb.propd_cache_observe(tree, z(1, **i32), z(1, 4, **i32), q, z(1, 4, 4), k, kt, rows, 0.1)
    with pytest.raises(TypeError):
        pb.propd_cache_evict(k, k.clone(), rows, 4, 0)
    with pytest.raises(TypeError):
        pb.propd_rotary(q, kt, z(32), z(1, 4, **i32))
    with pytest.raises(ValueError):
        pb.propd_grouped_attention(tree, q, k, k, z(1, 3, 4, 64), z(1, 3, 4, 64), rows.seq_lens, 0.1)
