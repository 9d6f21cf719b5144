"""The calls of a paged cache and sampled acceptance, marshalled natively and in Python: the same outputs, and the same errors for what is refused."""
import numpy as np
import pytest
import torch

from gpu_util import to_dev
from paged_util import dev_cache, make_case
from paper_2402_13485_amd import synth
from test_gpu_bounded_cache import dev_tree
from test_gpu_marshal import both, flat
from test_gpu_parity import pb  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,codes", [("bf16", True), ("f32", False)])
def test_marshalling_in_python_is_the_same(pb, monkeypatch, dtype, codes):
    rng = np.random.default_rng(71)
    x = make_case(rng, dtype, codes, 4, 2, 64, [synth.chain_tree(9), synth.random_tree(rng, 9)], [40, 33], 16)
    tree, t = dev_tree(pb, x), {n: to_dev(x[n]) for n in ("q", "k_tree", "v_tree", "seq_lens")}
    tree.token = torch.randint(0, 50, tree.parent.shape, dtype=torch.int32, device="cuda")
    rand = lambda *s: torch.rand(s, device="cuda")
    logits, draft = (torch.randn((2, 9, 50), device="cuda").to(t["q"].dtype) for _ in range(2))
    u, u_next, slopes, lse = rand(2, 9), rand(2), rand(4), rand(2, 4, 9)
    i32 = dict(dtype=torch.int32, device="cuda")
    length, path, nxt = torch.tensor([3, 1], **i32), torch.tensor([[0, 1, 2, 0]] * 2, **i32), torch.tensor([5, 6], **i32)
    big = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    base = dev_cache(pb, x)

    def cache(**kw):
        c = pb.PagedCache(*(None if v is None else v.clone() for v in (base.k_pages, base.v_pages, base.page_table, base.k_scale, base.v_scale)))
        for n, v in kw.items():
            setattr(c, n, v)
        return c
    att = lambda c=None, **k: pb.propd_paged_attention(tree, t["q"], c or base, t["k_tree"], t["v_tree"], t["seq_lens"], 0.125, **k)

    def as_bytes(c):
        return [v.view(torch.uint8) if v.dtype == torch.float8_e4m3fn else v for v in vars(c).values() if v is not None]

    def commit(c=None, a=(length, path, nxt), **k):
        c, lens = c or cache(), t["seq_lens"].clone()
        return [pb.propd_paged_commit(tree, *a, t["k_tree"], t["v_tree"], c, lens, **k), *as_bytes(c), lens, *k.values()]

    def prompt(c=None, k=t["k_tree"], v=t["v_tree"], lens=None, **kw):
        c, lens = c or cache(), t["seq_lens"].clone() if lens is None else lens
        pb.propd_paged_prompt(k, v, c, lens, **kw)
        return [*as_bytes(c), lens, *kw.values()]
    read = lambda c=None, k=None, v=None, **kw: pb.propd_paged_read(c or base, t["seq_lens"], torch.zeros_like(t["k_tree"]) if k is None else k,
                                                                    torch.zeros_like(t["k_tree"]) if v is None else v, **kw)
    sampled = lambda **k: pb.propd_accept_sampled(tree, logits, u, u_next, **k)
    zeros = lambda: torch.zeros(2, **i32)
    good = [lambda: att(out=torch.zeros_like(t["q"])), lambda: att(want_lse=True, out=torch.zeros_like(t["q"]), cap=5.0, window=9, slopes=slopes, lse=torch.zeros_like(lse)),
            lambda: att(out=torch.zeros_like(t["q"]), lse=torch.zeros_like(lse), workspace=big), commit, lambda: commit(seq_lens_out=zeros()),
            lambda: commit(out_stride=2)[:-1], prompt, lambda: prompt(n_rows=length), lambda: prompt(n_rows=length, seq_lens_out=zeros()), read,
            lambda: read(first=length), sampled, lambda: sampled(path_stride=2, inv_temperature=2), lambda: sampled(draft_logits=draft, draft_inv_temperature=0.5, workspace=big)]
    for n, call in enumerate(good):
        native, python = both(pb, monkeypatch, call)
        assert type(native) is type(python), (n, native, python)
        native, python = flat(native), flat(python)
        assert len(native) == len(python) > 0, n
        for a, b in zip(native, python):
            assert a.shape == b.shape and a.dtype == b.dtype and a.contiguous().view(torch.uint8).equal(b.contiguous().view(torch.uint8)), n
    for call in (lambda: att(want_lse=True), att):  # outputs made by the call
        native, python = both(pb, monkeypatch, call)
        assert [z.shape for z in flat(native)] == [z.shape for z in flat(python)]
    cpu = {k: v.cpu() for k, v in t.items()}
    bad = [lambda: att(cap=-1.0), lambda: att(window=-1), lambda: att(window=1.5), lambda: att(slopes=slopes[:3]), lambda: att(lse=lse.cpu()), lambda: att(out=t["q"]),
           lambda: att(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), lambda: att(cache(page_table=base.page_table[:1])), lambda: att(cache(v_pages=base.v_pages[1:])),
           lambda: att(cache(k_pages=base.k_pages[0])), lambda: att(out=base.k_pages.view(torch.uint8).flatten()[:t["q"].nbytes].view(t["q"].dtype).view(t["q"].shape)),
           lambda: commit(out_stride=-1), lambda: commit(out_stride="7"), lambda: commit(a=(length, path[0], nxt)), lambda: commit(a=(length.long(), path, nxt)),
           lambda: commit(seq_lens_out=length), lambda: prompt(k=t["k_tree"].half(), v=t["v_tree"].half()), lambda: prompt(k=cpu["k_tree"], v=cpu["v_tree"]),
           lambda: prompt(v=t["v_tree"][:1]), lambda: prompt(n_rows=length[:1]), lambda: prompt(cache(v_pages=base.k_pages, k_pages=base.k_pages)),
           lambda: prompt(k=t["k_tree"][0], v=t["v_tree"][0]), lambda: read(v=t["k_tree"], k=t["k_tree"]), lambda: read(first=length.float()),
           lambda: sampled(inv_temperature=0.0), lambda: sampled(inv_temperature="1"), lambda: sampled(draft_logits=draft[:1]), lambda: sampled(path_stride=0),
           lambda: sampled(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), lambda: pb.propd_accept_sampled(tree, logits[0], u, u_next),
           lambda: pb.propd_accept_sampled(tree, logits, u.double(), u_next)]
    if codes:
        bad += [lambda: att(cache(k_scale=None)), lambda: prompt(cache(k_scale=base.v_scale, v_scale=base.v_scale)), lambda: read(cache(v_scale=base.v_scale.int()))]
    for n, call in enumerate(bad):
        native, python = both(pb, monkeypatch, call)
        assert isinstance(native, Exception) and type(native) is type(python) and str(native) == str(python), (n, native, python)
