"""Weights of the cache's attention that are far below a row's largest, against closed forms
in 64 bits."""

from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import kv_ref as R  # noqa: E402
from gpu_util import DEV  # noqa: E402
from paper_2607_18253_amd import PagedKV  # noqa: E402

BF, F16, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def sink_case(q_len, hq, hkv, d, dtype, cache, C, seed=0):
    """A first key with a score of 16 to 18 and C - 1 others with 0, in pages that all the
    sequences share: (handle, pages, table, q, scores of the first key, V's held rows)."""
    S, T = 64, sum(q_len)
    g = torch.Generator().manual_seed(seed)
    kv = PagedKV(hq, hkv, d, block_size=S, dtype=dtype, cache_dtype=cache, max_seqs=len(q_len), max_tokens=max(T, C))
    pages = kv.new_pages(C // S)
    k = torch.zeros((C, hkv, d), dtype=dtype)
    k[0, :, 0] = 16.0
    v = (0.5 + 0.5 * torch.rand((C, hkv, d), generator=g)).to(dtype)
    v[0] = 0.0
    one = torch.randperm(C // S, generator=g).int()[None].to(DEV)
    kv.plan([C], [C])
    kv.append(pages, k.to(DEV), v.to(DEV), one)
    q = torch.randn((T, hq, d), generator=g).to(dtype)
    first = (8.0 + torch.rand((T, hq), generator=g)).to(dtype)   # times 16 times the scale 1/8
    q[:, :, 0] = first
    held = kv.read(pages, one)[1]
    kv.plan(q_len, [C] * len(q_len))
    return kv, pages, one.expand(len(q_len), -1).contiguous(), q.to(DEV), 2.0 * first.double().to(DEV), held.double()


@pytest.mark.parametrize("lse", [False, True])
@pytest.mark.parametrize("cache", [F16, E4])
@pytest.mark.parametrize("q_len,hq,hkv", [([1] * 256, 16, 8), ([1024], 64, 1)])
def test_weights_far_below_the_largest(q_len, hq, hkv, cache, lse):
    """One key 16 to 18 above 32767 others: each of these weighs 2^-23 to 2^-26 of it, all
    together a thousandth.  Few tiles of many sequences, and a chunk's tiles, are whole: one
    running maximum for all keys.

    out = e^-s sum_j v_j / (1 + (n - 1) e^-s).  Each weight is off by its rounding to 16 bits, u
    and at most 2^-36 of the largest one's, the scores by one product's rounding (their only
    one: 2^-24 of 18, as the argument of exp), the exponential by 2^-21, the result by u."""
    C, d = 32768, 64
    kv, pages, tab, q, s, v = sink_case(q_len, hq, hkv, d, F16, cache, C)
    z = torch.empty(q.shape[:2], device=DEV) if lse else None
    out = kv.attend(pages, q, tab, scale=0.125, lse=z).double()
    kv.sync()
    n = torch.cat([torch.arange(C - m + 1, C + 1, device=DEV) for m in q_len])   # keys that a row sees
    total = torch.cumsum(v, 0)[n - 1].repeat_interleave(hq // hkv, dim=1)           # of V: [T][hq][d]
    w = torch.exp(-s)
    norm = 1.0 + (n[:, None] - 1) * w
    want = total * (w / norm)[..., None]
    u = R.U[F16]
    rel = 2 * u + 2 * (18.0 * 2.0 ** -24 + 2.0 ** -21)
    bound = want * rel * 1.01 + n[:, None, None] * 2.0 ** -36 + 2.0 ** -25
    bad = (out - want).abs() > bound
    assert not bad.any(), (int(bad.sum()), float((out / want - 1).abs().max()))
