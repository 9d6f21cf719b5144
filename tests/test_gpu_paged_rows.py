"""Rows to and from the pages of a paged cache on the GPU against oracle/paged_cache.py: every bit, and every byte that has to stay."""
import numpy as np
import pytest
import torch

from cache_util import f64
from gpu_util import sentinel_like, to_dev, to_host
from oracle import paged_cache as ref
from paged_util import codes_as_bits, numbers
from paper_2402_13485_amd import synth
from test_gpu_parity import dev_tree, pb  # noqa: F401

pytestmark = pytest.mark.gpu

TYPES = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]


def empty_pool(rng, dtype, codes, Hk, d, B, table_pages, R):
    """A table in any order over recognisable contents."""
    n_pages = B * table_pages + 2
    table = rng.permutation(n_pages)[:B * table_pages].reshape(B, table_pages).astype(np.int32)
    shape = (n_pages, Hk, R, d)
    x = dict(page_table=table, k_scale=None, v_scale=None)
    for name in "kv":
        if codes:
            x[name + "_pages"], x[name + "_scale"] = np.full(shape, 0x4d, np.uint8), np.full(shape[:3], 0x4d, np.uint8)
        else:
            x[name + "_pages"] = sentinel_like(numbers(rng, dtype, *shape))
    return x


def dev_pool(pb, x):
    codes = x["k_scale"] is not None
    pages = [torch.from_numpy(x[n]).cuda().view(torch.float8_e4m3fn) if codes else to_dev(x[n]) for n in ("k_pages", "v_pages")]
    return pb.PagedCache(*pages, to_dev(x["page_table"]), *((to_dev(x["k_scale"]), to_dev(x["v_scale"])) if codes else ()))


def expect(x, rows, taken, seq_lens):
    """-> dict of arrays after the rows were appended, new lengths"""
    want = {}
    for name in "kv":
        scales = x[name + "_scale"]
        pages = np.array(x[name + "_pages"]) if scales is not None else np.array(x[name + "_pages"]).astype(np.float64) if x[name + "_pages"].dtype == np.float32 else None
        source = rows[name]
        if scales is not None:
            want[name + "_scale"] = np.array(scales)
            lens = ref.append(f64(source), taken, pages, want[name + "_scale"], x["page_table"], seq_lens)
            want[name + "_pages"] = pages
        else:  # bits
            pages = np.array(x[name + "_pages"])
            lens = ref.append(source, taken, pages, None, x["page_table"], seq_lens)
            want[name + "_pages"] = pages
    return want, lens


def check_pool(cache, want):
    for name, a in want.items():
        t = getattr(cache, name)
        got = codes_as_bits(t) if t.dtype == torch.float8_e4m3fn else to_host(t)
        same = got == a
        if got.dtype == np.float32:
            same |= np.isnan(got) & np.isnan(a)
        assert same.all(), (name, np.argwhere(~same)[:5], got[~same][:5], a[~same][:5])


def special_rows(rows, dtype):
    """Zeros, ties, numbers that are not finite, the largest and the least ones, minus zero."""
    x = synth.as_float(rows).astype(np.float32)
    flat = x.reshape(-1, x.shape[-1])
    n = len(flat)
    flat[0 % n] = 0
    flat[1 % n, :4] = [np.inf, -np.inf, np.nan, 448.0]
    flat[2 % n] = np.nan
    flat[3 % n] *= np.float32(1e38) / np.abs(flat[3 % n][np.isfinite(flat[3 % n])]).max(initial=1.0)
    flat[4 % n, :3] = [3.38e38, -3.38e38, 2.9e38]
    flat[5 % n] *= np.float32(1e-38)
    flat[6 % n] = np.float32(1e-40)
    flat[7 % n] = np.arange(len(flat[0])) / 16 * np.where(np.arange(len(flat[0])) % 2, 1, -1)  # ties, minus zero
    flat[8 % n, 0] = 448.0
    flat[8 % n, 1:] = np.clip(flat[8 % n, 1:], -1, 1)
    flat[9 % n, :2] = [450.0, -0.0]
    return synth.from_float(x, dtype)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d,R", [(64, 16), (128, 32), (128, 1024)])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_commit(pb, dtype, codes, d, R, in_place):
    """Paths of one node to many over page borders, entries that are no nodes, lengths out of range, a full sequence, missing pages."""
    rng = np.random.default_rng(d + R + codes)
    B, Hk, T, stride, table_pages = 7, 3, 40, 9, 3 if R < 1024 else 1
    room = table_pages * R
    x = empty_pool(rng, dtype, codes, Hk, d, B, table_pages, R)
    n_nodes = np.array([40, 5, 40, 1, 40, 40, 17], np.int32)
    parent = np.tile(np.arange(-1, T - 1, dtype=np.int32), (B, 1))
    token = rng.integers(0, 1000, (B, T)).astype(np.int32)
    rows = {name: special_rows(numbers(rng, dtype, B, Hk, T, d), dtype) for name in "kv"}
    lens = np.array([0, R - 1, room - 4, R - 3, room, -5, 10 ** 6], np.int32)
    a = np.array([9, 3, 7, 1, 2, 12, -1], np.int32)
    path = np.sort(rng.integers(0, T, (B, stride)).astype(np.int32), 1)
    path[:, 0] = 0
    path[1, :3] = [0, 4, 5]      # not a node of a tree of 5
    path[0, 3], path[0, 5] = -1, 40
    if table_pages > 1:
        x["page_table"][5, 0] = -1
    nxt = rng.integers(0, 1000, B).astype(np.int32)
    cache, seq = dev_pool(pb, x), to_dev(lens)
    out = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    tree = dev_tree(pb, n_nodes, parent, token)
    tokens = pb.propd_paged_commit(tree, to_dev(a), to_dev(path), to_dev(nxt), to_dev(rows["k"]), to_dev(rows["v"]), cache, seq, out_stride=8,
                                   seq_lens_out=None if in_place else out)
    torch.cuda.synchronize()
    taken = [[int(i) if 0 <= i < n_nodes[b] else None for i in path[b, :min(max(a[b], 0), stride)]] for b in range(B)]
    want, want_lens = expect(x, rows, taken, lens)
    check_pool(cache, want)
    assert to_host(seq if in_place else out).tolist() == want_lens.tolist()
    if not in_place:
        assert to_host(seq).tolist() == lens.tolist()
    assert to_host(cache.page_table).tolist() == x["page_table"].tolist()
    want_tokens = np.full((B, 8), -1)
    for b, t in enumerate(taken):
        line = [-1 if i is None else token[b, i] for i in t[1:]] + ([nxt[b]] if t else [])
        want_tokens[b, :min(len(line), 8)] = line[:8]
    assert to_host(tokens).tolist() == want_tokens.tolist()


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("S,Hk,d,R", [(1, 1, 64, 16), (37, 2, 128, 16), (300, 3, 64, 64), (700, 2, 128, 128)])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_prompts(pb, dtype, codes, S, Hk, d, R, in_place):
    """One row to several workgroups' worth, ragged, behind rows that are there, and more than fit."""
    rng = np.random.default_rng(S + codes)
    B, table_pages = 3, -(-(S + 20) // R)
    x = empty_pool(rng, dtype, codes, Hk, d, B, table_pages, R)
    rows = {name: numbers(rng, dtype, B, Hk, S, d) for name in "kv"}
    lens, n = np.array([0, 13, table_pages * R - min(S, 5)], np.int32), np.array([S, max(S - 9, 0), 10 ** 6], np.int32)
    cache, seq, out = dev_pool(pb, x), to_dev(lens), torch.full((B,), -7, dtype=torch.int32, device="cuda")
    pb.propd_paged_prompt(to_dev(rows["k"]), to_dev(rows["v"]), cache, seq, n_rows=to_dev(n), seq_lens_out=None if in_place else out)
    torch.cuda.synchronize()
    taken = [list(range(min(max(int(m), 0), S))) for m in n]
    if S > 100:  # (the float64 definition takes 10 us per value: whole rows by the library's cast, which it is pinned to)
        want, want_lens = expect_fast(x, rows, taken, lens)
    else:
        want, want_lens = expect(x, rows, taken, lens)
    check_pool(cache, want)
    assert to_host(seq if in_place else out).tolist() == want_lens.tolist()


def expect_fast(x, rows, taken, lens):
    quantise = ref.quantise

    def cast(row):
        most = np.abs(row).max()
        power = int(np.ceil(np.log2(most / 448)))
        return torch.from_numpy((row / 2.0 ** power).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), power + 127
    try:
        ref.quantise = cast
        return expect(x, rows, taken, lens)
    finally:
        ref.quantise = quantise


def test_prompt_without_row_counts(pb):
    rng = np.random.default_rng(4)
    x = empty_pool(rng, "bf16", True, 2, 64, 2, 4, 16)
    rows = {name: numbers(rng, "bf16", 2, 2, 20, 64) for name in "kv"}
    lens = np.array([3, 40], np.int32)
    cache, seq = dev_pool(pb, x), to_dev(lens)
    pb.propd_paged_prompt(to_dev(rows["k"]), to_dev(rows["v"]), cache, seq)
    want, want_lens = expect(x, rows, [list(range(20))] * 2, lens)
    check_pool(cache, want)
    assert to_host(seq).tolist() == want_lens.tolist()


@pytest.mark.parametrize("with_first", [True, False])
@pytest.mark.parametrize("S,Hk,d,R", [(1, 1, 64, 16), (37, 2, 128, 16), (150, 3, 64, 64), (300, 2, 128, 1024)])
@pytest.mark.parametrize("dtype,codes", TYPES)
def test_read(pb, dtype, codes, S, Hk, d, R, with_first):
    """Every row that is there, zeros where there is no page, and nothing else; every code among the values."""
    rng = np.random.default_rng(S + codes)
    B, table_pages = 4, -(-(S + 40) // R)
    n_pages = B * table_pages
    table = rng.permutation(n_pages).reshape(B, table_pages).astype(np.int32)
    lens = np.array([S, min(S + 33, table_pages * R), 0, 10 ** 6], np.int32)
    first = np.array([0, 7, 0, -3], np.int32) if with_first else np.zeros(B, np.int32)
    if table_pages > 1:
        table[1, 1] = n_pages
    shape = (n_pages, Hk, R, d)
    pages, scales, values = {}, {}, {}
    for name in "kv":
        if codes:
            pages[name], scales[name] = rng.integers(0, 256, shape).astype(np.uint8), rng.integers(10, 247, shape[:3]).astype(np.uint8)
            values[name] = ref.decode(pages[name], scales[name])
        else:
            pages[name] = numbers(rng, dtype, *shape)
            values[name] = f64(pages[name])
    dev = [torch.from_numpy(pages[n]).cuda().view(torch.float8_e4m3fn) if codes else to_dev(pages[n]) for n in "kv"]
    cache = pb.PagedCache(*dev, to_dev(table), *((to_dev(scales["k"]), to_dev(scales["v"])) if codes else ()))
    blank = sentinel_like(numbers(rng, dtype, B, Hk, S, d))
    k, v = pb.propd_paged_read(cache, to_dev(lens), to_dev(blank), to_dev(blank), first=to_dev(first) if with_first else None)
    torch.cuda.synchronize()
    room = table_pages * R
    for name, got in (("k", to_host(k)), ("v", to_host(v))):
        all_rows, _ = ref.dense(values[name], table, np.minimum(lens, room), room)
        want = f64(blank)
        for b in range(B):
            f, L = max(int(first[b]), 0), min(int(lens[b]), room)
            m = min(S, max(L - f, 0))
            want[b, :, :m] = all_rows[b, :, f:f + m]
        # values are exact: bf16 and fp32 hold a code times its scale
        assert np.array_equal(f64(got), want, equal_nan=True), name


def test_written_rows_are_read_back(pb):
    """Within half a step of the 8-bit type: 2^-4 of a value, or of the row's least normal one."""
    rng = np.random.default_rng(6)
    x = empty_pool(rng, "bf16", True, 2, 128, 1, 8, 16)
    rows = [numbers(rng, "bf16", 1, 2, 100, 128) for _ in range(2)]
    cache, seq = dev_pool(pb, x), torch.zeros(1, dtype=torch.int32, device="cuda")
    pb.propd_paged_prompt(to_dev(rows[0]), to_dev(rows[1]), cache, seq)
    k, v = (torch.zeros((1, 2, 100, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pb.propd_paged_read(cache, seq, k, v)
    for got, r in ((k, rows[0]), (v, rows[1])):
        r = f64(r)
        least = np.abs(r).max(-1, keepdims=True) / 224 * 2.0 ** -6  # a scale is at most the largest value over 224
        assert (np.abs(f64(to_host(got)) - r) <= 2.0 ** -4 * np.maximum(np.abs(r), least)).all()


def test_large_batches_and_long_prompts_share_the_workgroups(pb):
    """More rows than a workgroup takes at once, in place: the lengths are written behind all that read them."""
    B, Hk, S, d, R = 40, 8, 600, 128, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((B, Hk, S, d), generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(B * 20, generator=gen, device="cuda").int().view(B, 20)
    pages = [torch.zeros((B * 20, Hk, R, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache, seq = pb.PagedCache(*pages, table), torch.arange(B, dtype=torch.int32, device="cuda")
    for _ in range(2):
        pb.propd_paged_prompt(k, v, cache, seq)
    assert seq.tolist() == [b + 2 * S for b in range(B)]
    first = torch.arange(B, dtype=torch.int32, device="cuda")
    for n in range(2):
        a, c = pb.propd_paged_read(cache, seq, torch.zeros_like(k), torch.zeros_like(v), first=first + n * S)
        assert torch.equal(a, k) and torch.equal(c, v)


def test_rows_beyond_32_bits(pb):
    """A pool of 9 GB of K and of V: rows to its last pages and back."""
    for dtype in (torch.float32, torch.float8_e4m3fn):
        R, Hk, d = 1024, 8, 128
        n_pages = (9 << 30) // (R * Hk * d * (4 if dtype == torch.float32 else 1)) + 2
        pages = [torch.zeros((n_pages, Hk, R, d), dtype=torch.uint8 if dtype != torch.float32 else dtype, device="cuda").view(dtype) for _ in range(2)]
        scales = [torch.full((n_pages, Hk, R), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if dtype != torch.float32 else ()
        cache = pb.PagedCache(*pages, torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda"), *scales)
        gen = torch.Generator(device="cuda").manual_seed(3)
        k, v = (torch.randint(-8, 9, (1, Hk, 1100, d), generator=gen, device="cuda").float() for _ in range(2))  # exact in 8 bits
        seq = torch.zeros(1, dtype=torch.int32, device="cuda")
        pb.propd_paged_prompt(k, v, cache, seq)
        a, b = pb.propd_paged_read(cache, seq, torch.zeros_like(k), torch.zeros_like(v))
        assert seq.tolist() == [1100] and torch.equal(a, k) and torch.equal(b, v)
        del pages, scales, cache
        torch.cuda.empty_cache()


def test_what_overlaps_or_disagrees_is_refused(pb):
    rng = np.random.default_rng(7)
    x = empty_pool(rng, "bf16", True, 2, 64, 2, 4, 16)
    cache, seq = dev_pool(pb, x), torch.zeros(3, dtype=torch.int32, device="cuda")
    lens = seq[:2]
    k, v = (to_dev(numbers(rng, "bf16", 2, 2, 5, 64)) for _ in range(2))
    replaced = lambda **kw: pb.PagedCache(**{**{n: getattr(cache, n) for n in ("k_pages", "v_pages", "page_table", "k_scale", "v_scale")}, **kw})
    for call in (lambda: pb.propd_paged_prompt(k, v, replaced(v_pages=cache.k_pages), lens), lambda: pb.propd_paged_prompt(k, v, replaced(v_scale=cache.k_scale), lens),
                 lambda: pb.propd_paged_prompt(k, v, replaced(v_scale=None), lens), lambda: pb.propd_paged_prompt(k, v, replaced(k_scale=cache.k_scale[:3]), lens),
                 lambda: pb.propd_paged_prompt(k, v, cache, lens, seq_lens_out=seq[1:]), lambda: pb.propd_paged_prompt(k, v[:, :1].contiguous(), cache, lens),
                 lambda: pb.propd_paged_prompt(k, v, replaced(page_table=cache.page_table[:1]), lens), lambda: pb.propd_paged_read(cache, lens, k, k),
                 lambda: pb.propd_paged_prompt(k, v, replaced(v_pages=cache.v_pages[1:]), lens), lambda: pb.propd_paged_prompt(k, v, cache, seq),
                 lambda: pb.propd_paged_prompt(k, v, replaced(k_pages=cache.k_pages[0]), lens), lambda: pb.propd_paged_read(cache, lens, k, v[:1])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pb.propd_paged_prompt(k.half(), v.half(), cache, lens), lambda: pb.propd_paged_prompt(k, v.float(), cache, lens),
                 lambda: pb.propd_paged_prompt(k, v, replaced(v_pages=cache.v_pages.view(torch.uint8)), lens), lambda: pb.propd_paged_prompt(k, v, cache, lens.long()),
                 lambda: pb.propd_paged_prompt(k.transpose(2, 3), v.transpose(2, 3), cache, lens), lambda: pb.propd_paged_prompt(k, v, replaced(page_table=cache.page_table.cpu()), lens)):
        with pytest.raises(TypeError):
            call()
    assert seq.tolist() == [0, 0, 0]
