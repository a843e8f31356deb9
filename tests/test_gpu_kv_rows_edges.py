"""Weights, selections and moves on the paged cache where batches leave the ordinary sizes: pages that a
window hides, contexts at the limit, many contexts, lists that go on behind their end."""

from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import kv_ref as R  # noqa: E402
from gpu_util import DEV  # noqa: E402
from paper_2607_18253_amd import PagedKV  # noqa: E402
from paper_2607_18253_amd import lar as L  # noqa: E402
from test_gpu_kv import BF, E4, F16, Batch, refused  # noqa: E402
from test_gpu_kv_rows import KINDS, KINDS_OF_WEIGHTS, Cache, check_select, run_weigh, weigh_ref  # noqa: E402
from test_kv_rows_host import tree  # noqa: E402


# ------------------------------------------------------------------ pages that a window hides
def unseen(table, q_len, ctx, S, window, sinks):
    """The table without the pages that no new token sees."""
    out = table.clone()
    for s, (n, c) in enumerate(zip(q_len, ctx)):
        low = max(0, c - n) - window + 1
        for i in range(-(-c // S)):
            if n and i * S >= sinks and (i + 1) * S <= low:
                out[s, i] = -1
    assert (out != table).any()
    return out


HIDDEN = [([70], [5000], 100, 4),          # a chunk
          ([1], [3001], 64, 0),            # one token
          ([1, 3, 200, 40, 0], [900, 700, 4000, 2000, 600], 90, 70),
          ([600, 1], [9000, 5000], 33, 300)]


@pytest.mark.parametrize("q_len,ctx,window,sinks", HIDDEN)
@pytest.mark.parametrize("S", [1, 16, 128])
@pytest.mark.parametrize("cache", [BF, E4])
def test_weigh_in_place_without_hidden_pages(q_len, ctx, window, sinks, S, cache):
    """Pages that a window hides from all new tokens may be gone: they are not looked at, and all other rows
    get what they get with them."""
    b = Batch(q_len, ctx, hq=8, hkv=2, d=64, S=S, dtype=BF, cache=cache)
    _, lse = b.attend(window, sinks)
    tab = unseen(b.table.cpu(), q_len, ctx, S, window, sinks)
    old = torch.rand((b.pages.k.shape[0], 2, S), generator=torch.Generator().manual_seed(1)).to(DEV)
    want, got = old.clone(), old.clone()
    b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), b.table, want)
    b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), tab.to(DEV), got)
    b.k.sync()
    assert torch.equal(got, want)
    gone = torch.unique(b.table.cpu()[tab != b.table.cpu()]).long().to(DEV)
    assert torch.equal(got[gone], old[gone])


@pytest.mark.parametrize("q_len,ctx,window,sinks", HIDDEN)
@pytest.mark.parametrize("S", [1, 16, 128])
def test_weigh_from_before_without_hidden_pages(q_len, ctx, window, sinks, S):
    """The same from weights that lie apart: what has no place is not carried over."""
    b = Batch(q_len, ctx, hq=8, hkv=2, d=128, S=S, dtype=F16, cache=F16)
    _, lse = b.attend(window, sinks)
    tab = unseen(b.table.cpu(), q_len, ctx, S, window, sinks)
    old = torch.rand((b.pages.k.shape[0], 2, S), generator=torch.Generator().manual_seed(1)).to(DEV)
    want, got = torch.full_like(old, 9.0), torch.full_like(old, 9.0)
    b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), b.table, want, before=old)
    b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), tab.to(DEV), got, before=old)
    b.k.sync()
    gone = torch.unique(b.table.cpu()[tab != b.table.cpu()]).long().to(DEV)
    assert torch.equal(want[gone], old[gone])
    want[gone] = 9.0
    assert torch.equal(got, want)


@pytest.mark.parametrize("place", [True, False])
def test_weigh_reports_lost_pages_that_are_seen(place):
    """Under a window too, for chunks and single tokens, in the window and among the sinks."""
    q_len, ctx, window, sinks, S = [70, 1], [2000, 900], 100, 20, 16
    b = Batch(q_len, ctx, hq=8, hkv=2, d=64, S=S, dtype=BF, cache=BF)
    _, lse = b.attend(window, sinks)
    for s, i in ((0, 0), (0, (2000 - 70 - 99) // S), (0, 1999 // S), (1, 1), (1, 800 // S), (1, 899 // S)):
        tab = b.table.clone()
        tab[s, i] = -1
        w = b.k.new_weights(b.pages.k.shape[0])
        b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), tab, w if place else torch.empty_like(w), before=None if place else w)
        refused(L.LAR_E_STATE, b.k.sync)
        b.k.plan(q_len, ctx, window=window, sinks=sinks)
        b.k.sync()


@pytest.mark.parametrize("ctx", [40000000, (1 << 29) + 77, 1 << 30])
@pytest.mark.parametrize("G,q_len", [(64, 40), (64, 1), (8, 3), (8, 90)])
@pytest.mark.parametrize("place", [True, False])
def test_weigh_far_from_the_sinks(ctx, G, q_len, place):
    """The longest contexts under a window: only the pages of sinks and window are there."""
    window, sinks, S, d = 300, 5, 65536, 64
    cols, low = -(-ctx // S), ctx - q_len - window + 1
    kv = PagedKV(G, 1, d, block_size=S, dtype=BF, max_seqs=1, max_tokens=1000)
    pages = kv.new_pages(4)
    tab = torch.full((1, cols), -1, dtype=torch.int32)
    tab[0, 0], tab[0, low // S], tab[0, cols - 1] = 2, 0, 0 if low // S == cols - 1 else 3
    g = torch.Generator().manual_seed(G)
    for t in pages.tensors():
        t.zero_()
    rows = []
    for n, end in ((sinks, sinks), (ctx - low, ctx)):
        k = torch.randn((n, 1, d), generator=g).to(BF)
        kv.plan([n], [end])
        kv.append(pages, k.to(DEV), k.to(DEV), tab.to(DEV))
        rows.append(k)
    k = torch.cat(rows).double()
    at = torch.cat([torch.arange(sinks), torch.arange(low, ctx)])
    q = torch.randn((q_len, G, d), generator=g).to(BF)
    p = torch.arange(ctx - q_len, ctx)[:, None]
    mask = (at <= p) & ((at > p - window) | (at < sinks))
    s = torch.einsum("thd,jd->htj", q.double(), k[:, 0]) * d ** -0.5
    lse = torch.logsumexp(torch.where(mask, s, -torch.inf), 2).T.float().contiguous()
    old = torch.rand((4, 1, S), generator=g)
    want, bound = weigh_ref(SimpleNamespace(q_len=[q_len], ctx=[ctx], d=d, held=[[k]], q=q), 0, 0, mask, lse, d ** -0.5,
                            torch.where(at < ctx - q_len, old[tab[0].long()[at // S], 0, at % S].double(), 0.0)[:, None])
    kv.plan([q_len], [ctx], window=window, sinks=sinks)
    w = old.to(DEV)
    new = w if place else torch.full_like(w, 9.0)
    kv.weigh(pages, q.to(DEV), lse.to(DEV), tab.to(DEV), new, before=None if place else w)
    kv.sync()
    got = new.cpu()[tab[0].long()[at // S], 0, at % S].double()[:, None]
    assert ((got - want).abs() <= bound).all(), float(((got - want).abs() / bound).max())
    # page 0 past the sinks is carried over as it was; page 1 is no one's
    assert torch.equal(new.cpu()[2, 0, sinks:], old[2, 0, sinks:])
    assert torch.equal(new.cpu()[1], old[1] if place else torch.full_like(old[1], 9.0))


# ------------------------------------------------------------------ kernels by the number of key blocks
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,cache", KINDS)
def test_weigh_of_many_key_blocks(dtype, cache, d):
    """More than 256 blocks of keys and heads: 64 keys for a wave, no rows shared out."""
    run_weigh([40], [9000], hq=16, hkv=8, d=d, dtype=dtype, cache=cache)
    run_weigh([40, 33, 1, 70], [5003, 3000, 90, 1000], hq=40, hkv=8, d=d, dtype=dtype, cache=cache, place=False)


# ------------------------------------------------------------------ selections by the number of contexts
def lengths(at, most, n, seed):
    """n lengths, among them those around multiples of `at`."""
    rng = np.random.RandomState(seed)
    near = [k * at + e for k in (1, 2, 3, most // at) for e in (-1, 0, 1) if k * at + e <= most]
    return near + [int(c) for c in np.exp(rng.uniform(0, np.log(most), n - len(near)))]


@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (64, 4, 16), (513, 0, 0), (1000, 4, 128)])
def test_select_of_some_hundred_contexts(budget, first, last):
    """512 threads for a context of up to 16384 rows."""
    check_select(lengths(512, 16384, 100, budget), budget, first, last, hkv=3, seed=budget)


@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (64, 4, 16), (255, 0, 255), (1000, 4, 128)])
@pytest.mark.parametrize("most", [2048, 2049])
def test_select_of_many_contexts(budget, first, last, most):
    """256 threads for a context of up to 2048 rows, 512 from 2049 on."""
    check_select(lengths(256, 2048, 359, budget) + [most], budget, first, last, hkv=3, seed=budget)


@pytest.mark.parametrize("kind", sorted(KINDS_OF_WEIGHTS))
@pytest.mark.parametrize("ctx,hkv", [([70000], 1), ([5000, 4097, 2500] * 30, 3), ([1500, 400, 2048, 900] * 90, 3)])
def test_select_values_in_every_kernel(kind, ctx, hkv):
    """A context that is cut, and those of 512 and 256 threads."""
    for budget, first, last in ((50, 3, 20), (333, 0, 1)):
        check_select(ctx, budget, first, last, hkv=hkv, make=KINDS_OF_WEIGHTS[kind])


def test_select_of_more_rows_than_fit():
    """Contexts that a workgroup reads again for every digit: more rows in all than the working memory of
    cut ones has, and one of more stretches than are cut."""
    make = lambda r, s: r.randint(0, 300, s).astype(np.float32)  # noqa: E731
    check_select([40000] * 110, 777, 4, 60, hkv=2, make=make, S=64)
    for kind in ("not finite", "neighbours"):
        check_select([(1 << 20) + 4097], 90000, 4, 60, hkv=1, make=KINDS_OF_WEIGHTS[kind], S=64)


# ------------------------------------------------------------------ lists that go on behind their end
@pytest.mark.parametrize("end", [32, 64, 128, 256, 512, 1024, 2048])
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("cache", [BF, E4])
def test_entries_behind_a_lists_end_are_reported(end, weights, cache):
    """Wherever the first -1 is, and however far behind it another entry."""
    x = Cache([1, 1], [3000, 2600], cache=cache)
    for more in (1, 7, 400):
        n = end + more + 1
        rows = np.full((2, 2, n), -1, np.int32)
        rows[:, :, :end] = np.arange(end)
        x.kv.plan([1, 1], [3000, 2600])
        x.kv.keep(x.pages, x.tab.to(DEV), torch.from_numpy(rows).to(DEV), weights=x.w if weights else None)
        x.kv.sync()
        rows[1, 1, n - 1] = 2500
        x.kv.keep(x.pages, x.tab.to(DEV), torch.from_numpy(rows).to(DEV), weights=x.w if weights else None)
        refused(L.LAR_E_STATE, x.kv.sync)


# ------------------------------------------------------------------ trees at the limit
@pytest.mark.parametrize("ctx", [(1 << 29) + 77, 1 << 30])
@pytest.mark.parametrize("G,q_len", [(64, 40), (8, 4), (4, 300)])
def test_trees_far_from_the_sinks(ctx, G, q_len):
    """The longest contexts under a window, of which only the pages of sinks and window are there."""
    window, sinks, S, d = 300, 5, 65536, 64
    cols, low = -(-ctx // S), ctx - q_len - window + 1
    kv = PagedKV(G, 1, d, block_size=S, dtype=BF, max_seqs=1, max_tokens=1000)
    pages = kv.new_pages(4)
    tab = torch.full((1, cols), -1, dtype=torch.int32)
    tab[0, 0], tab[0, low // S], tab[0, cols - 1] = 2, 0, 0 if low // S == cols - 1 else 3
    for t in pages.tensors():
        t.zero_()
    g = torch.Generator().manual_seed(G)
    # keys from the first page of attention's tile of 64 with the window's start on
    start = low // 64 * 64
    rows = []
    for n, end in ((sinks, sinks), (ctx - start, ctx)):
        kv.plan([n], [end])
        k, v = (torch.randn((n, 1, d), generator=g).to(BF) for _ in range(2))
        kv.append(pages, k.to(DEV), v.to(DEV), tab.to(DEV))
        rows.append((k, v))
    k, v = (torch.cat([r[i] for r in rows]).double() for i in range(2))
    at = torch.cat([torch.arange(sinks), torch.arange(start, ctx)])
    par = tree(q_len, np.random.RandomState(G))
    places, line = [], []
    for i, a in enumerate(par):
        places.append(ctx - q_len + (0 if a < 0 else places[a] - (ctx - q_len) + 1))
        line.append(([] if a < 0 else line[a]) + [i])
    mask = torch.zeros((q_len, len(at)), dtype=torch.bool)
    for i in range(q_len):
        where = torch.where(at < ctx - q_len, at, -1)
        for x in line[i]:
            where[len(at) - q_len + x] = places[x]
        mask[i] = (where >= 0) & ((where > places[i] - window) | (where < sinks))
    q = (2.0 * torch.randn((q_len, G, d), generator=g)).to(BF)
    kv.plan([q_len], [ctx], window=window, sinks=sinks, parents=par)
    lse = torch.empty((q_len, G), dtype=torch.float32, device=DEV)
    out = kv.attend(pages, q.to(DEV), tab.to(DEV), lse=lse)
    kv.sync()
    want, wz, mag, big = R.attend_fast(q.double(), k, v, mask, d ** -0.5)
    bo, bz = R.bounds(BF, mag, big, wz, d, len(at), float(v.abs().max()))
    Batch.near(out.cpu().double(), want, bo, ctx)
    Batch.near(lse.cpu().double(), wz, bz, (ctx, "lse"))
