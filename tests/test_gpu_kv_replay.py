"""Captured calls of the paged cache replayed while another batch is planned."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from gpu_util import DEV  # noqa: E402
from test_gpu_kv import BF, E4, Batch, bits, refused  # noqa: E402
from paper_2607_18253_amd import lar as L  # noqa: E402


@pytest.mark.parametrize("q_len,ctx", [([1, 60, 2], [2000, 500, 33]), ([1, 1, 1], [3000, 40, 7])])
@pytest.mark.parametrize("other", [([1, 60, 2], [2001, 500, 33]), ([1], [5]), ([300], [300]), ([1] * 3, [2000, 500, 33])])
@pytest.mark.parametrize("cache", [BF, E4])
def test_replay_under_another_plan(q_len, ctx, other, cache):
    """It writes nothing, neither pages nor results, and the next sync reports it; under its own
    plan, made anew, it runs again."""
    T = sum(q_len)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = Batch(q_len, ctx, hq=8, hkv=2, d=128, S=16, dtype=BF, cache=cache, spare=200)
        want, _ = b.attend(lse=False)
        q, out = b.q.to(DEV), torch.full(b.q.shape, 3.0, dtype=BF, device=DEV)
        k, v = (torch.randn((T, 2, 128), device=DEV).to(BF) for _ in range(2))
        ko, vo = torch.full_like(k, 5.0), torch.full_like(v, 5.0)
        b.k.append(b.pages, k, v, b.table)
        want = b.k.attend(b.pages, q, b.table).clone()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.k.append(b.pages, k, v, b.table)
            b.k.attend(b.pages, q, b.table, out=out)
            b.k.read(b.pages, b.table, ko, vo)
        k0 = k.clone()
        for turn in range(2):
            b.k.plan(*other)
            k.copy_(-k0)
            out.fill_(3.0)
            ko.fill_(5.0)
            before = [t.clone() for t in b.pages.tensors()]
            graph.replay()
            refused(L.LAR_E_STATE, b.k.sync)
            assert (out == 3.0).all() and (ko == 5.0).all()
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(b.pages.tensors(), before))
            k.copy_(k0)
            b.k.plan(q_len, ctx)
            graph.replay()
            b.k.sync()
            assert torch.equal(bits(out), bits(want))
            assert torch.isfinite(ko.float()).all()
