"""Attention without the log of the sums, the form that a caller gets by default and that has
kernels of its own for chunks, and the precision of single tokens."""

from __future__ import annotations

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import kv_ref as R  # noqa: E402
from gpu_util import DEV  # noqa: E402
from test_gpu_kv import BF, E4, F16, Batch, bits  # noqa: E402
from paper_2607_18253_amd import PagedKV  # noqa: E402

TYPES = [(BF, BF), (F16, F16), (BF, E4), (F16, E4)]


def both(b, window=0, sinks=0):
    """The results with the log-sums, checked against the definition, and those without: the
    weights and their sums are the same, and so is every bit."""
    b.check(window, sinks)
    with_lse, _ = b.attend(window, sinks)
    without, _ = b.attend(window, sinks, lse=False)
    assert torch.equal(bits(with_lse), bits(without))


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 128), (8, 2, 64), (5, 1, 64), (16, 2, 128), (64, 1, 64)])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_lengths(hq, hkv, d, dtype, cache):
    both(Batch([1, 64, 1, 33, 200, 1, 70], [33, 64, 500, 33, 1200, 0, 60], hq=hq, hkv=hkv, d=d, S=16, dtype=dtype, cache=cache,
               seed=hq))


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (64, 64), (100, 4), (33, 200)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_windows(window, sinks, d, dtype, cache):
    both(Batch([3, 80, 200, 1, 40], [301, 400, 200, 97, 1000], hq=8, hkv=2, d=d, S=16, dtype=dtype, cache=cache), window, sinks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_split_chunks(d, dtype, cache):
    """A chunk whose keys are split over workgroups and joined."""
    both(Batch([100], [9000], hq=4, hkv=1, d=d, S=16, dtype=dtype, cache=cache))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_long_chunk(d, dtype, cache):
    """One whose workgroups walk over the same keys; the definition on the GPU, rows in blocks."""
    hq, S, n, c = 4, 16, 2049, 70017
    kv = PagedKV(hq, 1, d, block_size=S, dtype=dtype, cache_dtype=cache, max_seqs=1, max_tokens=c)
    g = torch.Generator(device=DEV).manual_seed(4)
    k, v = (torch.randn((c, 1, d), device=DEV, generator=g).to(dtype) for _ in range(2))
    q = (2 * torch.randn((n, hq, d), device=DEV, generator=g)).to(dtype)
    blocks = -(-c // S)
    tab = torch.randperm(blocks, device=DEV, generator=g).int()[None].contiguous()
    pages = kv.new_pages(blocks)
    kv.plan([c], [c])
    kv.append(pages, k, v, tab)
    k, v = kv.read(pages, tab)
    kv.plan([n], [c])
    out = kv.attend(pages, q, tab)
    kv.sync()
    kk, vv = k[:, 0].double(), v[:, 0].double()
    for h in range(hq):
        for a in (0, 1024, n - 300):
            b = a + 300
            mask = R.sees(b - a, c - n + b).to(DEV)
            m = mask.shape[1]
            want, wz, mag, big = R.attend_fast(q[a:b, h:h + 1].double(), kk[:m, None], vv[:m, None], mask, d ** -0.5)
            bo, _ = R.bounds(dtype, mag, big, wz, d, c, float(vv.abs().max()))
            Batch.near(out[a:b, h:h + 1].double(), want.to(DEV), bo.to(DEV), (h, a))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F16])
def test_single_tokens_weigh_in_more_than_16_bits(d, dtype):
    """On a 16-bit cache a single token's weights go into the product in two parts: off by 2^-16 of
    themselves (bf16: 2 x 8 bits), not by the type's u.  Seen where V's values cancel: the result's own
    rounding, u of it, is small against u of the magnitudes.

    Scores are off by (d + 2) 2^-24 of their magnitudes and the exponentials' argument, as in kv_ref;
    the sum of the weights as much."""
    n_seq, ctx, hq, hkv = 40, 24, 8, 2
    u, extra = R.U[dtype], 2.0 ** -15 + 2.0 ** -18

    def edit(b, rows):
        for k, v in rows:
            k *= 0.25
            v.copy_(torch.sign(v) + torch.where(v == 0, 1.0, 0.0).to(v.dtype))
            v[1::2] = -v[::2]
    b = Batch([1] * n_seq, [ctx] * n_seq, hq=hq, hkv=hkv, d=d, S=16, dtype=dtype, cache=dtype, edit=edit)
    out, _ = b.attend(lse=False)
    seen = 0
    for s in range(n_seq):
        k, v = b.held[s]
        mask = R.sees(1, ctx)
        want, _, mag, big = R.attend_fast(b.q[s:s + 1].double(), k, v, mask, d ** -0.5)
        ds = (d + 2) * 2.0 ** -24 * big
        bound = 1.01 * u * want.abs() + (extra + 2 * torch.expm1(ds))[..., None] * mag + 2.0 ** -25
        Batch.near(out[s:s + 1].double(), want, bound, s)
        # the same with weights rounded to the type: the bound tells it apart
        for h in range(hq):
            x = (k[:, h // (hq // hkv)] @ b.q[s, h].double()) * d ** -0.5
            w = torch.exp(x - x.max()).to(dtype).double()
            one = (w @ v[:, h // (hq // hkv)]) / w.sum()
            seen += int(((one.to(dtype).double() - want[0, h]).abs() > bound[0, h]).sum())
    assert seen > 0


def test_rows_of_any_pitch_for_one_token():
    """One token's rows out of a tensor with an odd pitch: that stride reaches no second token."""
    b = Batch([1], [70], hq=8, hkv=2, d=64, S=16, dtype=BF, cache=BF)
    want, _ = b.attend(lse=False)
    flat = torch.zeros(3 * 517, dtype=BF, device=DEV)
    q = flat.as_strided((1, 8, 64), (517, 64, 1))
    q.copy_(b.q.to(DEV))
    assert torch.equal(bits(b.k.attend(b.pages, q, b.table).cpu()), bits(want))
    k, v = b.k.read(b.pages, b.table)
    k2 = flat.as_strided((1, 2, 64), (517, 64, 1), 1024)
    k2.copy_(k)
    b.k.append(b.pages, k2, v, b.table)
    assert torch.equal(bits(b.k.attend(b.pages, q, b.table).cpu()), bits(want))


def test_rows_that_share_memory_and_gradients_are_refused():
    from paper_2607_18253_amd import LarError
    b = Batch([3, 1], [70, 5], hq=8, hkv=2, d=64, S=16, dtype=BF, cache=BF)
    b.k.plan([3, 1], [70, 5])
    new = torch.empty((4, 2, 64), dtype=BF, device=DEV)
    fused = torch.empty((4, 4, 64), dtype=BF, device=DEV)
    for k, v in ((new[:1].expand(4, 2, 64), new), (new, new[:, :1].expand(4, 2, 64)), (new, new), (fused[:, :2], fused[:, 1:3])):
        with pytest.raises(LarError):
            b.k.read(b.pages, b.table, k, v)
    k, v = b.k.read(b.pages, b.table)
    b.k.read(b.pages, b.table, fused[:, :2], fused[:, 2:])
    assert torch.equal(bits(fused[:, :2]), bits(k)) and torch.equal(bits(fused[:, 2:]), bits(v))
    q = b.q.to(DEV).requires_grad_()
    with pytest.raises(ValueError):
        b.k.attend(b.pages, q, b.table)
    with torch.no_grad():
        got = b.k.attend(b.pages, q, b.table)
    assert torch.equal(bits(got), bits(b.k.attend(b.pages, q.detach(), b.table)))
    b.k.sync()


def test_plan_while_another_stream_captures():
    """On a handle of the default stream: refused, and the capture goes on."""
    from paper_2607_18253_amd import LarError
    kv = PagedKV(8, 2, 64, block_size=16, max_seqs=1, max_tokens=4)
    x = torch.zeros(4, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        with pytest.raises(LarError):
            kv.plan([1], [4])
        x.add_(1.0)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert (x == 3.0).all()
    kv.plan([1], [4])
    kv.sync()
