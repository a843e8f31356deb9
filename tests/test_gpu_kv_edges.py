"""Edges of the paged cache's calls: values that are not finite in sight of a row, scales and
tensors at the ends of what a call takes."""

from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import kv_ref as R  # noqa: E402
from test_gpu_kv import BF, F16, Batch  # noqa: E402


@pytest.mark.parametrize("q_len,ctx,G", [([1], [200], 4), ([1, 2], [2000, 33], 8), ([7], [9000], 4), ([40, 300], [600, 300], 4)])
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 20)])
def test_visible_infinities(q_len, ctx, G, dtype, window, sinks):
    """Infinities in V wherever a context has them: a row that sees them is infinite, or NaN
    where both signs or a NaN meet, and its other values are as ever."""
    def edit(b, rows):
        for k, v in rows:
            c = len(v)
            k *= 0.25
            v[0, 0, 1] = math.inf
            v[c // 2, 0, 2] = -math.inf
            v[c // 3, 1, 3] = math.inf
            v[c // 3, 0, 4], v[c - 1, 0, 4] = math.inf, -math.inf
            v[min(40, c - 1), 1, 5] = math.nan
    b = Batch(q_len, ctx, hq=2 * G, hkv=2, d=64, S=16, dtype=dtype, cache=dtype, edit=edit)
    b.q *= 0.25   # every key has some weight
    for lse in (True, False):
        out, z = b.attend(window, sinks, lse=lse)
        at = 0
        for s, (n, c) in enumerate(zip(q_len, ctx)):
            k, v = b.held[s]
            mask = R.sees(n, c, window, sinks)
            want, wz, _, _ = R.attend(b.q[at:at + n].double(), k, v, mask, 0.125)
            fin = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
            w2, _, mag, big = R.attend(b.q[at:at + n].double(), k, fin, mask, 0.125)
            bo, bz = R.bounds(dtype, mag, big, wz, 64, c, 8.0)
            got = out[at:at + n].double()
            Batch.near(got, torch.where(torch.isfinite(want), w2, want), bo, (s, n, c))
            if lse:
                Batch.near(z[at:at + n].double(), wz, bz, (s, "lse"))
            at += n


@pytest.mark.parametrize("n", [1, 50])
@pytest.mark.parametrize("scale", [1e-40, 1e-60, 5e-324])
def test_smallest_scales(n, scale):
    """Scales that 32 bits hold only just or not at all: every key that a row sees weighs the same."""
    b = Batch([n], [77], hq=8, hkv=2, d=64, S=16, dtype=BF, cache=BF)
    b.check(scale=scale)
