"""Inputs of the calls of a paged cache: host arrays, with NaN wherever nothing may be read."""
import numpy as np
import torch

from cache_util import f64, make_inputs
from gpu_util import to_dev
from oracle import paged_cache as ref
from paper_2402_13485_amd import synth


def numbers(rng, dtype, *shape, scale=1.0):
    return synth.from_float((rng.normal(size=shape) * scale).astype(np.float32), dtype)


def codes_of(rng, *shape):
    """Random codes as rows of N(0,1) have them"""
    x = torch.from_numpy(np.clip(rng.normal(size=shape) * 128, -448, 448).astype(np.float32))
    return x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def make_pool(rng, dtype, codes, Hk, d, lens, R, extra_rows=0, spare=3):
    """Pages in any order for sequences of these lengths; NaN in the pages of nobody and behind the sequences.
    -> dict of page_table, k_pages, v_pages (bits), k_scale, v_scale (None without codes), k64, v64 (values)"""
    B = len(lens)
    table_pages = max(1, -(-(max(lens) + extra_rows) // R))
    n_pages = B * table_pages + spare
    table = rng.permutation(n_pages)[:B * table_pages].reshape(B, table_pages).astype(np.int32)
    used = np.zeros((n_pages, R), bool)
    for b, L in enumerate(lens):
        for j in range(L):
            used[table[b, j // R], j % R] = True
    x = dict(page_table=table, R=R)
    for name in "kv":
        if codes:
            c, s = codes_of(rng, n_pages, Hk, R, d), rng.integers(118, 122, (n_pages, Hk, R)).astype(np.uint8)
            c = np.where(used[:, None, :, None], c, 0x7f).astype(np.uint8)
            x[name + "_pages"], x[name + "_scale"], x[name + "64"] = c, s, ref.decode(c, s)
        else:
            c = numbers(rng, dtype, n_pages, Hk, R, d)
            nan = np.uint16(0x7fc0) if dtype == "bf16" else np.float32(np.nan)
            x[name + "_pages"] = np.where(used[:, None, :, None], c, nan)
            x[name + "_scale"], x[name + "64"] = None, f64(x[name + "_pages"])
    return x


def dev_cache(pb, x):
    codes = x["k_scale"] is not None
    pages = [torch.from_numpy(x[n]).cuda().view(torch.float8_e4m3fn) if codes else to_dev(x[n]) for n in ("k_pages", "v_pages")]
    return pb.PagedCache(*pages, to_dev(x["page_table"]), *((to_dev(x["k_scale"]), to_dev(x["v_scale"])) if codes else ()))


def make_case(rng, dtype, codes, H, Hk, d, shapes, lens, R, T_max=None, sigma=1.0):
    """The tensors of a tree (cache_util.make_inputs) and a pool"""
    x = make_inputs(rng, dtype, H, Hk, d, shapes, [0] * len(lens), T_max=T_max, sigma=sigma)
    x.update(make_pool(rng, dtype, codes, Hk, d, lens, R), seq_lens=np.array(lens, np.int32))
    return x


def codes_as_bits(t):
    return t.view(torch.uint8).cpu().numpy()
