"""What the calls of a paged cache and sampled acceptance refuse, on the host, before anything is enqueued (no GPU needed)."""
import ctypes
import math

import pytest
import torch

from test_abi import pb  # noqa: F401

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
OK, ODD = 0x1000, 0x1004  # never dereferenced: validation fails first


def tree_of(pb, B=2, T_max=16, **ptr):
    a = dict(n_nodes=OK, parent=OK, token=OK, depth=OK, anc=OK)
    a.update(ptr)
    return ctypes.byref(pb._Tree(B, T_max, a["n_nodes"], a["parent"], a["token"], a["depth"], a["anc"]))


def cache_of(pb, dt=1, n_pages=8, table_pages=4, page_rows=16, **ptr):
    a = dict(k=OK, v=OK, ks=OK, vs=OK, table=OK)
    a.update(ptr)
    return ctypes.byref(pb._PagedCache(a["k"], a["v"], a["ks"], a["vs"], a["table"], dt, n_pages, table_pages, page_rows))


def attention(pb, dt=1, H=8, H_kv=2, d=128, tree=None, cache=None, scale=0.1, cap=0.0, window=0, ws=OK, ws_bytes=1 << 40, **ptr):
    a = dict(q=OK, kt=OK, vt=OK, lens=OK, out=OK)
    a.update(ptr)
    return pb.load_library().propd_paged_attention(tree or tree_of(pb), dt, H, H_kv, d, ctypes.byref(pb._ScoreRule(scale, cap, window, None)), a["q"],
                                                   cache or cache_of(pb, dt), a["kt"], a["vt"], a["lens"], a["out"], None, ws, ws_bytes, None)


def commit(pb, dt=1, H_kv=2, d=128, tree=None, cache=None, stride=8, out_stride=8, **ptr):
    a = dict(len=OK, path=OK, next=OK, kt=OK, vt=OK, lens=OK, lens_out=OK, tokens=OK)
    a.update(ptr)
    return pb.load_library().propd_paged_commit(tree or tree_of(pb), dt, H_kv, d, a["len"], a["path"], stride, a["next"], a["kt"], a["vt"],
                                                cache or cache_of(pb, dt), a["lens"], a["lens_out"], a["tokens"], out_stride, None)


def prompt(pb, dt=1, B=2, S=5, H_kv=2, d=128, cache=None, **ptr):
    a = dict(n=None, k=OK, v=OK, lens=OK, lens_out=OK)
    a.update(ptr)
    return pb.load_library().propd_paged_prompt(dt, B, S, H_kv, d, a["n"], a["k"], a["v"], cache or cache_of(pb, dt), a["lens"], a["lens_out"], None)


def read(pb, dt=1, B=2, S=5, H_kv=2, d=128, cache=None, **ptr):
    a = dict(k=OK, v=OK, lens=OK)
    a.update(ptr)
    return pb.load_library().propd_paged_read(dt, B, S, H_kv, d, cache or cache_of(pb, dt), a["lens"], None, a["k"], a["v"], None)


CALLS = dict(attention=attention, commit=commit, prompt=prompt, read=read)


@pytest.mark.parametrize("name", list(CALLS))
def test_caches_that_are_refused(pb, name):
    call = CALLS[name]
    for dt in (pb.PROPD_BF16, pb.PROPD_F32):
        for ptr in ("k", "v"):
            assert call(pb, dt, cache=cache_of(pb, dt, **{ptr: None})) == INVALID and call(pb, dt, cache=cache_of(pb, dt, **{ptr: ODD})) == INVALID
        assert call(pb, dt, cache=cache_of(pb, dt, table=None)) == INVALID
        assert call(pb, dt, cache=cache_of(pb, pb.PROPD_E4M3, ks=None)) == INVALID and call(pb, dt, cache=cache_of(pb, pb.PROPD_E4M3, vs=None)) == INVALID
        for kw in (dict(n_pages=0), dict(table_pages=0), dict(page_rows=0), dict(page_rows=8), dict(page_rows=24), dict(page_rows=2048), dict(page_rows=-16)):
            assert call(pb, dt, cache=cache_of(pb, dt, **kw)) == INVALID, kw
        assert call(pb, dt, cache=cache_of(pb, dt, table_pages=(1 << 26) + 1)) == UNSUPPORTED
        assert call(pb, dt, d=96) == UNSUPPORTED and call(pb, dt, d=256) == UNSUPPORTED
        assert call(pb, dt, H_kv=0) == INVALID
    assert call(pb, pb.PROPD_BF16, cache=cache_of(pb, pb.PROPD_F32)) == INVALID and call(pb, pb.PROPD_F32, cache=cache_of(pb, pb.PROPD_BF16)) == INVALID
    assert call(pb, pb.PROPD_E4M3, cache=cache_of(pb, pb.PROPD_E4M3)) == INVALID and call(pb, 7, cache=cache_of(pb, 1)) == INVALID


def test_attention_refusals(pb):
    for dt in (pb.PROPD_BF16, pb.PROPD_F32):
        assert attention(pb, dt, ws=None) == WORKSPACE and attention(pb, dt, ws_bytes=100) == WORKSPACE
        assert attention(pb, dt, H=8, H_kv=3) == INVALID and attention(pb, dt, H=0) == INVALID
        for name in ("q", "kt", "vt", "out"):
            assert attention(pb, dt, **{name: ODD}) == INVALID and attention(pb, dt, **{name: None}) == INVALID, name
        assert attention(pb, dt, ws=ODD) == INVALID and attention(pb, dt, lens=None) == INVALID
        for kw in (dict(T_max=129), dict(T_max=0), dict(B=0), dict(anc=None), dict(anc=0x1008), dict(n_nodes=None)):
            assert attention(pb, dt, tree=tree_of(pb, **kw)) == INVALID, kw
        assert attention(pb, dt, tree=tree_of(pb, B=(1 << 20) + 1)) == UNSUPPORTED
    for scale, cap, window in ((0.0, 0.0, 0), (-1.0, 0.0, 0), (math.nan, 0.0, 0), (math.inf, 0.0, 0), (1.0, -1.0, 0), (1.0, math.nan, 0), (1.0, 2e3, 0),
                               (1.0, 0.0, -1), (1.0, 0.0, (1 << 24) + 1)):
        assert attention(pb, scale=scale, cap=cap, window=window) == INVALID


def test_row_refusals(pb):
    for name in ("len", "path", "kt", "vt", "lens", "lens_out", "next"):
        assert commit(pb, **{name: None}) == INVALID, name
    assert commit(pb, kt=ODD) == INVALID and commit(pb, vt=ODD) == INVALID
    assert commit(pb, stride=0) == INVALID and commit(pb, out_stride=0) == INVALID
    for kw in (dict(T_max=129), dict(T_max=0), dict(B=0), dict(n_nodes=None), dict(token=None)):
        assert commit(pb, tree=tree_of(pb, **kw)) == INVALID, kw
    assert commit(pb, tree=tree_of(pb, B=65536)) == UNSUPPORTED and commit(pb, stride=1 << 30, H_kv=4) == UNSUPPORTED
    for name in ("k", "v", "lens", "lens_out"):
        assert prompt(pb, **{name: None}) == INVALID, name
    assert prompt(pb, k=ODD) == INVALID and prompt(pb, v=ODD) == INVALID and prompt(pb, S=0) == INVALID and prompt(pb, B=0) == INVALID
    assert prompt(pb, B=65536) == UNSUPPORTED and prompt(pb, S=1 << 30, H_kv=4) == UNSUPPORTED
    for name in ("k", "v", "lens"):
        assert read(pb, **{name: None}) == INVALID, name
    assert read(pb, k=ODD) == INVALID and read(pb, S=0) == INVALID and read(pb, B=0) == INVALID and read(pb, B=8192, H_kv=8) == UNSUPPORTED


def sampled(pb, dt=1, vocab=100, inv=1.0, draft=None, draft_inv=1.0, stride=8, ws=OK, ws_bytes=1 << 40, tree=None, **ptr):
    a = dict(logits=OK, u=OK, u_next=OK, len=OK, path=OK, next=OK)
    a.update(ptr)
    return pb.load_library().propd_accept_sampled(tree or tree_of(pb), dt, vocab, a["logits"], inv, draft, draft_inv, a["u"], a["u_next"], a["len"], a["path"],
                                                  stride, a["next"], ws, ws_bytes, None)


def test_sampled_refusals(pb):
    for name in ("logits", "u", "u_next", "len", "path", "next"):
        assert sampled(pb, **{name: None}) == INVALID, name
    for kw in (dict(vocab=0), dict(stride=0), dict(dt=2), dict(dt=7), dict(inv=0.0), dict(inv=-1.0), dict(inv=math.nan), dict(inv=math.inf), dict(inv=2.0 ** 21),
               dict(draft=OK, draft_inv=0.0), dict(draft=OK, draft_inv=math.nan), dict(ws=ODD)):
        assert sampled(pb, **kw) == INVALID, kw
    for kw in (dict(T_max=129), dict(T_max=0), dict(B=0), dict(n_nodes=None), dict(parent=None), dict(token=None)):
        assert sampled(pb, tree=tree_of(pb, **kw)) == INVALID, kw
    assert sampled(pb, vocab=(1 << 20) + 1) == UNSUPPORTED and sampled(pb, tree=tree_of(pb, B=(1 << 21) + 1)) == UNSUPPORTED
    assert sampled(pb, ws=None) == WORKSPACE and sampled(pb, ws_bytes=100) == WORKSPACE
    # a draft temperature is looked at only with a draft
    assert sampled(pb, draft_inv=0.0, ws=None) == WORKSPACE


def test_workspace_sizes(pb):
    assert pb.workspace_bytes(pb.WS_PAGED_ATTENTION, 2, 16, 8, 128, 64) > 0 and pb.workspace_bytes(pb.WS_PAGED_ATTENTION, 2, 16, 0, 128, 64) == 0
    assert pb.workspace_bytes(pb.WS_ACCEPT_SAMPLED, 2, 16, vocab=100) > 0 and pb.workspace_bytes(pb.WS_ACCEPT_SAMPLED, 2, 16, vocab=0) == 0
    assert pb.workspace_bytes(pb.WS_ACCEPT_SAMPLED, 2, 129, vocab=10) == 0


def test_tensors_in_host_memory_are_refused(pb):
    """No fallback: the binding takes tensors on the GPU only."""
    i32 = dict(dtype=torch.int32)
    tree = pb.Tree(torch.ones(1, **i32), -torch.ones((1, 4), **i32), token=torch.zeros((1, 4), **i32), anc=torch.ones((1, 4, 2), dtype=torch.int64))
    rows, pages = torch.zeros((1, 1, 4, 64)), torch.zeros((2, 1, 16, 64))
    cache = pb.PagedCache(pages, pages.clone(), torch.zeros((1, 2), **i32))
    one, path = torch.ones(1, **i32), torch.zeros((1, 4), **i32)
    for call in (lambda: pb.propd_paged_attention(tree, rows, cache, rows, rows, one, 0.1), lambda: pb.propd_paged_commit(tree, one, path, one, rows, rows, cache, one),
                 lambda: pb.propd_paged_prompt(rows, rows, cache, one), lambda: pb.propd_paged_read(cache, one, rows, rows.clone()),
                 lambda: pb.propd_accept_sampled(tree, torch.zeros((1, 4, 9)), torch.zeros((1, 4)), torch.zeros(1))):
        with pytest.raises(TypeError):
            call()


def test_other_calls_refuse_the_type_of_8_bit_pages(pb):
    lib, t, big = pb.load_library(), tree_of(pb), 1 << 40
    out = ctypes.byref(pb._TreeOut(OK, OK, OK, OK, OK))
    rule = ctypes.byref(pb._ScoreRule(0.1, 0.0, 0, None))
    rows = ctypes.byref(pb._CacheRows(OK, OK, OK, OK))
    e4m3 = pb.PROPD_E4M3
    for status in (lib.propd_tree_attention(t, e4m3, 2, 128, 1.0, OK, OK, OK, OK, OK, OK, 64, OK, OK, big, None),
                   lib.propd_early_prune(t, e4m3, 128, 1000, 4, OK, OK, OK, OK, OK, OK, OK, out, None, 0, None, OK, big, None),
                   lib.propd_early_prune_prob(t, e4m3, 128, 1000, 0, 0.5, 0, OK, OK, OK, OK, OK, OK, OK, out, None, 0, None, OK, big, None),
                   lib.propd_accept_path(t, e4m3, 100, OK, OK, OK, 8, OK, OK, big, None), lib.propd_accept_path_static(t, e4m3, 100, OK, OK, OK, 8, OK, None),
                   lib.propd_commit_path(t, e4m3, 2, 128, OK, OK, 8, OK, OK, OK, OK, OK, 64, OK, OK, 8, None),
                   lib.propd_grouped_attention(t, e4m3, 8, 2, 128, rule, OK, OK, OK, OK, OK, OK, None, None, 64, OK, None, OK, big, None),
                   lib.propd_cache_observe(t, e4m3, 8, 2, 128, rule, 0.5, OK, OK, 8, OK, OK, OK, OK, OK, None, None, OK, 64, None, OK, None),
                   lib.propd_cache_evict(2, e4m3, 2, 128, 64, 8, 1, 1, OK, 0x2000, rows, rows, OK, big, None),
                   lib.propd_rotary(e4m3, 2, 4, 2, 2, 64, 64, 0, 1, None, OK, None, OK, 1, None, OK, OK, OK, OK, None)):
        assert status == INVALID
