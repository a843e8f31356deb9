"""Trees of drafted tokens, weights, selections and moves on the paged cache (lar_kv_plan_tree, _weigh,
_select, _keep) against their definitions in 64 bits."""

from __future__ import annotations

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import kv_ref as R  # noqa: E402
from gpu_util import DEV  # noqa: E402
from paper_2607_18253_amd import PagedKV  # noqa: E402
from paper_2607_18253_amd import lar as L  # noqa: E402
from test_gpu_kv import BF, E4, F16, HEADS, Batch, bits, refused, table_for  # noqa: E402
from test_kv_rows_host import seen, tree  # noqa: E402

KINDS = [(BF, BF), (F16, F16), (BF, E4), (F16, E4)]


class Trees(Batch):
    """A batch whose sequences' new tokens have parents (one list for each)."""

    def __init__(self, q_len, ctx, parents, **kw):
        super().__init__(q_len, ctx, **kw)
        self.parents = parents

    def attend(self, window=0, sinks=0, scale=None, lse=True, q=None):
        self.k.plan(self.q_len, self.ctx, window=window, sinks=sinks, parents=sum(self.parents, []))
        q = self.q.to(DEV) if q is None else q
        z = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV) if lse else None
        out = torch.full(q.shape, 7.0, dtype=self.dtype, device=DEV)
        self.k.attend(self.pages, q, self.table, scale=scale, out=out, lse=z)
        self.k.sync()
        return out.cpu(), None if z is None else z.cpu()

    def mask(self, s, window=0, sinks=0):
        n, c = self.q_len[s], self.ctx[s]
        keys, _ = seen(self.parents[s], n, c, window, sinks)
        m = torch.zeros((n, c), dtype=torch.bool)
        for i, k in enumerate(keys):
            m[i, list(k)] = True
        return m

    def check(self, window=0, sinks=0, scale=None, fast=True, q=None):
        out, lse = self.attend(window, sinks, scale, q=q)
        scale = self.d ** -0.5 if scale is None else scale
        at = 0
        for s, (n, c) in enumerate(zip(self.q_len, self.ctx)):
            got, z = out[at:at + n].double(), lse[at:at + n].double()
            pad = min(n, max(0, n - c))
            assert (got[:pad] == 0).all() and (z[:pad] == -math.inf).all()
            if n > pad:
                k, v = self.held[s]
                f = R.attend_fast if fast else R.attend
                want, wz, mag, big = f(self.q[at + pad:at + n].double(), k, v, self.mask(s, window, sinks)[pad:], scale)
                bo, bz = R.bounds(self.dtype, mag, big, wz, self.d, c, float(v[torch.isfinite(v)].abs().max()))
                self.near(got[pad:], want, bo, (s, n, c))
                self.near(z[pad:], wz, bz, (s, n, c, "lse"))
            at += n


def trees(q_len, ctx, seed, spread=5):
    rng = np.random.RandomState(seed)
    out = []
    for n, c in zip(q_len, ctx):
        r0 = max(0, n - c)
        p = tree(n, rng, spread)
        out.append([-1 if i <= r0 or x < r0 else x for i, x in enumerate(p)])
    return out


# ------------------------------------------------------------------ trees
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype,cache", KINDS)
def test_tree_lengths(hq, hkv, d, dtype, cache):
    """Trees of a few and of many tokens, contexts around the tiles' and pages' ends, and none."""
    for q_len, ctx in (([2, 3, 2], [2, 35, 66]), ([5, 7, 8, 8], [37, 7, 40, 260]), ([16, 11, 3], [80, 11, 500]),
                       ([33, 64, 20, 1], [33, 64 + 31, 300, 9]), ([70, 130, 5], [71, 400, 64])):
        Trees(q_len, ctx, trees(q_len, ctx, hq), hq=hq, hkv=hkv, d=d, S=16, dtype=dtype, cache=cache, seed=hq).check()


@pytest.mark.parametrize("S", [1, 2, 64, 1024])
@pytest.mark.parametrize("cache", [BF, E4])
def test_tree_block_sizes(S, cache):
    q_len, ctx = [26, 7, 64], [77, 130, 1025]
    Trees(q_len, ctx, trees(q_len, ctx, S), hq=8, hkv=2, d=128, S=S, dtype=BF, cache=cache).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 0), (4, 3), (7, 300), (32, 0), (64, 64), (100, 4), (333, 200)])
@pytest.mark.parametrize("q_len", [[4, 8, 3], [16, 13, 2], [60, 90, 7]])
def test_tree_window(window, sinks, q_len):
    """Windows shorter than a tree is deep, and longer: they count places, not rows."""
    ctx = [q_len[0] + 300, q_len[1], q_len[2] + 95]
    for cache, d in ((F16, 64), (E4, 128)):
        Trees(q_len, ctx, trees(q_len, ctx, window, 3), hq=8, hkv=2, d=d, S=16, dtype=F16, cache=cache).check(window, sinks)


@pytest.mark.parametrize("cache", [BF, E4])
def test_trees_beside_other_sequences(cache):
    """Trees, single tokens, a chunk and empty slots in one batch, with and without a window; forests; padding
    rows in a tree."""
    q_len, ctx = [1, 20, 90, 6, 1, 0, 12, 1], [300, 320, 200, 70, 0, 40, 8, 33]
    par = trees(q_len, ctx, 5)
    par[2] = list(range(-1, 89))
    par[3] = [-1, -1, -1, 0, 2, 2]
    for w in ((0, 0), (50, 3)):
        Trees(q_len, ctx, par, hq=8, hkv=2, d=128, S=16, dtype=BF, cache=cache).check(*w)


@pytest.mark.parametrize("q,c,hkv", [(6, 20000, 1), (26, 9001, 2), (60, 30011, 1), (8, 4000, 8), (100, 6000, 2)])
@pytest.mark.parametrize("cache", [BF, E4])
def test_tree_split_contexts(q, c, hkv, cache):
    """One tree over a long context: the keys are split and the parts joined."""
    q_len, ctx = [q], [c]
    Trees(q_len, ctx, trees(q_len, ctx, q), hq=4 * hkv, hkv=hkv, d=128, S=16, dtype=BF, cache=cache).check()


def test_large_trees():
    """The largest trees, wide ones and deep ones."""
    for spread in (1000, 2):
        q_len, ctx = [1024, 300], [1500, 300]
        Trees(q_len, ctx, trees(q_len, ctx, 7, spread), hq=4, hkv=1, d=64, S=16, dtype=BF, cache=BF).check()


@pytest.mark.parametrize("q_len,G", [([3, 2], 4), ([7, 9], 4), ([30, 14], 4), ([70, 12], 8)])
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_tree_masked_values_have_no_part(q_len, G, dtype, bad):
    """Infinities and NaN in K and V of drafted tokens: only those below them see them, also through
    joins."""
    for more in (37, 6001):
        ctx = [n + more for n in q_len]
        par = trees(q_len, ctx, G, 1000)

        def edit(b, rows):
            for (k, v), n in zip(rows, q_len):
                v[-1, 0, 5] = bad
                v[-1, 0, 40] = -bad
                k[-1, 1, 3] = bad
                if n > 2:
                    v[-n // 2, 0, 11] = bad
        b = Trees(q_len, ctx, par, hq=2 * G, hkv=2, d=64, S=16, dtype=dtype, cache=dtype, edit=edit)
        out, lse = b.attend()
        at = 0
        for s, n in enumerate(q_len):
            mask = b.mask(s)
            want, wz, mag, big = R.attend(b.q[at:at + n].double(), *b.held[s], mask, 0.125)
            bo, bz = R.bounds(dtype, mag, big, wz, 64, ctx[s], 8.0)
            got = out[at:at + n].double()
            assert torch.equal(torch.isfinite(got), torch.isfinite(want)), s
            fin = torch.isfinite(want)
            assert (((got - want).abs() <= bo) | ~fin).all(), s
            clean = torch.isfinite(wz)
            assert (((lse[at:at + n].double() - wz).abs() <= bz) | ~clean).all(), s
            at += n


@pytest.mark.parametrize("cache", [BF, E4])
def test_chains_are_as_before(cache):
    """Parents that follow one another: the results of the plan without parents, bit for bit."""
    q_len, ctx = [1, 40, 3, 90], [300, 90, 900, 2000]
    b = Trees(q_len, ctx, [list(range(-1, n - 1)) for n in q_len], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=cache)
    x, z = b.attend()
    y, w = Batch.attend(b)
    assert torch.equal(bits(x), bits(y)) and torch.equal(z, w)


def test_tree_repeats_bit_for_bit():
    q_len, ctx = [20, 6, 1, 60], [3000, 20000, 70, 400]
    b = Trees(q_len, ctx, trees(q_len, ctx, 3), hq=8, hkv=2, d=128, S=16, dtype=BF, cache=BF)
    x, z = b.attend()
    for _ in range(3):
        y, w = b.attend()
        assert torch.equal(bits(x), bits(y)) and torch.equal(z, w)


# ------------------------------------------------------------------ weights
def weigh_ref(b, s, at, mask, lse, scale, old):
    """Weights of sequence s in 64 bits and how far they may be off; lse [n, hq] as given."""
    n, c, d = b.q_len[s], b.ctx[s], b.d
    k, G = b.held[s][0], b.q.shape[1] // b.held[s][0].shape[1]
    total, bound, rows = old.clone(), 2.0 ** -23 * old.abs(), n * G
    for h in range(b.q.shape[1]):
        q = b.q[at:at + n, h].double()
        x = (q @ k[:, h // G].T) * scale
        big = (q.abs() @ k[:, h // G].abs().T) * scale
        z = lse[:, h].double()[:, None]
        on = mask & (z != -math.inf)
        w = torch.where(on, torch.exp(x - z), 0.0)
        # scores as sums of d products in 32 bits; scale, product, log and difference rounded (in
        # log2 units, 2^-24 of each); the exponential 2^-21
        rel = torch.expm1((d + 2) * 2.0 ** -24 * big + 2.0 ** -24 * (2 * x.abs() + 2 * z.abs().nan_to_num(0, 0, 0) + (x - z).abs().nan_to_num(0, 0, 0))) + 2.0 ** -21
        total[:, h // G] += w.sum(0)
        bound[:, h // G] += torch.where(on, w * rel, 0.0).sum(0)
    # sums: 16 in a row, then one for every 32 rows, two halves, what was there
    bound += (20 + rows // 32) * 2.0 ** -24 * total.abs() + 1e-37 * rows
    return total, bound


def run_weigh(q_len, ctx, *, hq, hkv, d, S=16, dtype=BF, cache=BF, window=0, sinks=0, seed=0, place=True, scale=None,
              edit=None, lse_edit=None):
    b = Batch(q_len, ctx, hq=hq, hkv=hkv, d=d, S=S, dtype=dtype, cache=cache, seed=seed, edit=edit)
    scale_ = d ** -0.5 if scale is None else scale
    _, lse = b.attend(window, sinks, scale)
    if lse_edit:
        lse_edit(lse)
    n_blocks = b.pages.k.shape[0]
    old = torch.rand((n_blocks, hkv, S), generator=torch.Generator().manual_seed(seed + 1)) * 3
    w = old.to(DEV)
    if place:
        b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), b.table, w, scale=scale)
        rest = old
    else:
        new = torch.full_like(w, 9.0)
        b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), b.table, new, before=w, scale=scale)
        assert torch.equal(w.cpu(), old)
        w, rest = new, torch.full_like(old, 9.0)
    b.k.sync()
    got, at = w.cpu(), 0
    written = torch.zeros((n_blocks, S), dtype=torch.bool)
    for s, (n, c) in enumerate(zip(q_len, ctx)):
        if n and c:
            j = torch.arange(c)
            page, row = b.table[s].cpu().long()[j // S], j % S
            before = torch.where((j < c - n)[:, None], old[page, :, row].double(), 0.0)
            mask = torch.zeros((n, c), dtype=torch.bool)
            pad = max(0, n - c)
            mask[pad:] = R.sees(n - pad, c, window, sinks)
            want, bound = weigh_ref(b, s, at, mask, lse[at:at + n], scale_, before)
            yield_ = got[page, :, row].double()
            assert torch.equal(torch.isnan(yield_), torch.isnan(want)), (s, n, c)
            bad = ((yield_ - want).abs() > bound) & ~torch.isnan(want)
            assert not bad.any(), (s, n, c, int(bad.sum()), float(((yield_ - want).abs() / bound)[~torch.isnan(want)].max()))
            written[page, row] = True
        at += n
    keep = ~written
    assert torch.equal(got.transpose(1, 2)[keep], rest.transpose(1, 2)[keep])   # nothing else is touched
    return b


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype,cache", KINDS)
def test_weigh_lengths(hq, hkv, d, dtype, cache):
    q_len = [1, 1, 1, 1, 2, 3, 1, 5, 33, 64, 70, 9, 1, 0, 1]
    ctx = [1, 31, 32, 33, 64, 65, 500, 5, 33, 200, 129, 300, 96, 50, 97]
    run_weigh(q_len, ctx, hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, seed=hq)
    run_weigh([1, 1, 7], [90, 1, 300], hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, seed=hq, place=False)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (32, 0), (64, 64), (100, 4), (100, 90), (5000, 4), (33, 200)])
@pytest.mark.parametrize("place", [True, False])
def test_weigh_window(window, sinks, place):
    for cache, d in ((F16, 64), (E4, 128)):
        run_weigh([1, 1, 3, 80, 200, 1, 40], [1, 300, 301, 400, 200, 97, 1000], hq=8, hkv=2, d=d, dtype=F16, cache=cache,
                  window=window, sinks=sinks, place=place)


@pytest.mark.parametrize("S", [1, 2, 64, 1024])
@pytest.mark.parametrize("cache", [BF, E4])
def test_weigh_block_sizes_and_padding(S, cache):
    run_weigh([1, 2, 50, 1], [77, 130, 131, 1025], hq=8, hkv=2, d=128, S=S, cache=cache)
    run_weigh([5, 70, 2, 1], [3, 60, 0, 0], hq=8, hkv=2, d=128, S=S, cache=cache)
    run_weigh([300], [200], hq=8, hkv=2, d=128, S=S, cache=cache, window=40, sinks=3)


@pytest.mark.parametrize("q,c", [(1, 30000), (3, 9001), (700, 6000), (1500, 1501)])
def test_weigh_long(q, c):
    run_weigh([q], [c], hq=4, hkv=1, d=128)


def test_weigh_values_that_are_not_finite():
    """Keys that only later rows see; rows whose log-sum is -infinity add nothing; a NaN in a key makes
    the weights of the keys NaN whose rows it made so, no others'."""
    def edit(b, rows):
        rows[0][0][-1, 0, 3] = math.inf
        rows[1][0][-1, 1, 9] = math.nan
        rows[2][0][0, 0, 0] = -math.inf

    def lse_edit(z):
        z[0, 1] = -math.inf
        z[5, 3] = -math.inf
        z[48, 0] = math.inf
    run_weigh([5, 40, 1, 3], [60, 90, 50, 33], hq=8, hkv=2, d=64, edit=edit, lse_edit=lse_edit)


def test_weigh_weights_add_up_to_the_rows():
    """From nothing, a batch's weights add up to one for each row and head: over steps as over chunks."""
    ctx, hq, hkv, S = 700, 8, 2, 16
    b = Batch([ctx], [ctx], hq=hq, hkv=hkv, d=64, S=S, dtype=BF, cache=BF)
    q, lse = b.q.to(DEV), torch.empty((ctx, hq), dtype=torch.float32, device=DEV)
    whole, parts = b.k.new_weights(b.pages.k.shape[0]), b.k.new_weights(b.pages.k.shape[0])
    b.k.plan([ctx], [ctx])
    b.k.attend(b.pages, q, b.table, lse=lse)
    b.k.weigh(b.pages, q, lse, b.table, whole)
    at = 0
    for n in (300, 1, 1, 90, 2, 306):
        b.k.plan([n], [at + n])
        b.k.weigh(b.pages, q[at:at + n], lse[at:at + n], b.table, parts)
        at += n
    b.k.sync()
    # each weight is off by some 2^-18 of itself, so is a sum of them
    total = ctx * hq
    assert abs(float(whole.double().sum()) / total - 1) < 2.0 ** -16
    assert ((whole - parts).abs().double() <= 2.0 ** -16 * whole.double().abs() + 1e-6).all()


# ------------------------------------------------------------------ selection
def select_ref(w, budget, first, last):
    """Rows of weights w [c] (64 bits) to keep, by sorting."""
    c = len(w)
    if c <= budget:
        return list(range(c))
    j = np.arange(c)
    x = np.where(np.isnan(w), np.inf, w)
    must = (j < first) | (j >= c - last)
    return sorted(np.lexsort((j, -x, ~np.isnan(w), ~must))[:budget].tolist())


def check_select(ctx, budget, first, last, S=16, hkv=2, make=None, seed=0, q_len=None):
    rng = np.random.RandomState(seed)
    n_blocks = sum(-(-c // S) for c in ctx) + 2
    tab = table_for(ctx, S, n_blocks, rng)
    w = rng.randn(n_blocks, hkv, S).astype(np.float32) if make is None else make(rng, (n_blocks, hkv, S))
    q_len = [min(1, c) for c in ctx] if q_len is None else q_len
    kv = PagedKV(hkv, hkv, 64, block_size=S, dtype=BF, max_seqs=len(ctx), max_tokens=max(1, sum(q_len)))
    kv.plan(q_len, ctx)
    got = kv.select(torch.from_numpy(w).to(DEV), tab.to(DEV), budget, first, last)
    kv.sync()
    got, tab = got.cpu().numpy(), tab.numpy()
    for s, c in enumerate(ctx):
        j = np.arange(c)
        for h in range(hkv):
            want = select_ref(w[tab[s, j // S], h, j % S].astype(np.float64), budget, first, last)
            assert got[s, h].tolist() == want + [-1] * (budget - len(want)), (s, c, h)


@pytest.mark.parametrize("budget,first,last", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (2, 1, 1), (64, 4, 16), (65, 0, 0), (100, 100, 0),
                                               (100, 0, 100), (1000, 4, 128), (1024, 0, 1000), (5000, 16, 1)])
def test_select_lengths(budget, first, last):
    check_select([1, 2, 63, 64, 65, 66, 100, 101, 1000, 1023, 1024, 1025, 1026, 5001, 9000], budget, first, last)


@pytest.mark.parametrize("S", [1, 2, 64, 1024])
def test_select_block_sizes_and_sequences_without_tokens(S):
    check_select([0, 300, 77, 1300, 5], 60, 3, 10, S=S, hkv=3, q_len=[0, 0, 1, 2, 0])
    check_select([0, 300, 77, 1300, 5], 60, 3, 10, S=S, hkv=3, q_len=[0, 0, 0, 0, 0])


@pytest.mark.parametrize("c,budget", [(40000, 8192), (131072, 4096), (131071, 131000), (200003, 7)])
def test_select_long(c, budget):
    check_select([c, 50], budget, min(4, budget), min(500, budget - min(4, budget)), hkv=1)


KINDS_OF_WEIGHTS = {
    "equal": lambda r, s: np.full(s, 0.25, np.float32),
    "zeros of both signs": lambda r, s: np.where(r.rand(*s) < 0.5, 0.0, -0.0).astype(np.float32),
    "few values": lambda r, s: r.randint(-2, 3, s).astype(np.float32),
    "neighbours": lambda r, s: (1 + r.randint(0, 4, s) * 2.0 ** -23).astype(np.float32),
    "subnormal": lambda r, s: (r.randint(-3, 4, s) * 1e-45).astype(np.float32),
    "not finite": lambda r, s: r.choice(np.array([np.inf, -np.inf, np.nan, -np.nan, 1.0, -1.0, 3e38, -3e38], np.float32), s),
    "ascending": lambda r, s: np.arange(np.prod(s), dtype=np.float32).reshape(s),
    "wide range": lambda r, s: np.exp(r.randn(*s) * 30).clip(0, 3e38).astype(np.float32),
}


@pytest.mark.parametrize("kind", sorted(KINDS_OF_WEIGHTS))
def test_select_values(kind):
    for budget, first, last in ((50, 0, 0), (50, 3, 20), (333, 0, 1)):
        check_select([49, 51, 400, 1500], budget, first, last, make=KINDS_OF_WEIGHTS[kind])


# ------------------------------------------------------------------ moves
class Cache:
    """Random bytes in pages and weights, and the lists applied to copies of them."""

    def __init__(self, q_len, ctx, *, hkv=2, d=64, S=16, dtype=BF, cache=BF, spare=0, seed=0, parents=None):
        self.q_len, self.ctx, self.hkv, self.S = q_len, ctx, hkv, S
        self.rng = np.random.RandomState(seed)
        self.n_blocks = sum(-(-c // S) for c in ctx) + spare + 3
        self.tab = table_for(ctx, S, self.n_blocks, self.rng)
        self.kv = PagedKV(hkv, hkv, d, block_size=S, dtype=dtype, cache_dtype=cache, max_seqs=len(ctx),
                          max_tokens=max(1, sum(q_len)))
        self.pages = self.kv.new_pages(self.n_blocks)
        g = torch.Generator().manual_seed(seed)
        for t in self.pages.tensors():
            x = t.view(torch.uint8)
            x.copy_(torch.randint(0, 256, x.shape, dtype=torch.uint8, generator=g))
        self.w = torch.rand((self.n_blocks, hkv, S), generator=g).to(DEV)
        self.kv.plan(q_len, ctx, parents=parents)

    def tensors(self, weights):
        return [t.view(torch.uint8) for t in self.pages.tensors()] + ([self.w] if weights else [])

    def check(self, lists, new=False, to=None, weights=True, per_head=True):
        """lists[s][h] of positions."""
        heads = self.hkv if per_head else 1
        n = max([1] + [len(x) for s in lists for x in s])
        rows = np.full((len(lists), heads, n), -1, np.int32)
        for s, per in enumerate(lists):
            for h in range(heads):
                rows[s, h, :len(per[h])] = per[h]
        want = [t.clone() for t in self.tensors(True)]
        old = [t.clone() for t in want]
        dst = self.tab if to is None else to
        for s, per in enumerate(lists):
            base = self.ctx[s] - self.q_len[s] if new else 0
            for h in range(self.hkv):
                j = torch.tensor(per[h if per_head else 0], dtype=torch.long)
                if not len(j):
                    continue
                src, put = base + j, max(0, base) + torch.arange(len(j))
                a, b = self.tab[s].long()[src // self.S], dst[s].long()[put // self.S]
                for x, y in list(zip(old, want))[:None if weights else -1]:
                    y[b, h, put % self.S] = x[a, h, src % self.S]
        r = torch.from_numpy(rows if per_head else rows[:, 0].copy()).to(DEV)
        self.kv.keep(self.pages, self.tab.to(DEV), r, new=new, to=None if to is None else to.to(DEV),
                     weights=self.w if weights else None)
        self.kv.sync()
        for x, y in zip(self.tensors(True), want):
            assert torch.equal(x, y)


def some(rng, c, n):
    return sorted(rng.choice(c, min(n, c), replace=False).tolist())


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("weights", [True, False])
def test_keep_in_place(dtype, cache, d, weights):
    """Lists of any length, dense ones whose sources are other rows' places, and none."""
    ctx = [1, 5, 300, 64, 0, 2000, 777]
    x = Cache([min(1, c) for c in ctx], ctx, hkv=3, d=d, dtype=dtype, cache=cache)
    for turn in range(2):
        lists = [[some(x.rng, c, int(x.rng.choice([0, 1, c // 7, c // 2, c]))) for _ in range(3)] for c in ctx]
        x.check(lists, weights=weights)
    x.check([[list(range(1, c)) for _ in range(3)] for c in ctx], weights=weights)        # all one down
    x.check([[list(range(c // 2, c)) for _ in range(3)] for c in ctx], weights=weights)


@pytest.mark.parametrize("S", [1, 4, 64, 1024])
def test_keep_long(S):
    """More rows than a workgroup moves at once, in place."""
    ctx = [9000, 5000]
    x = Cache([1, 0], ctx, hkv=1, S=S, d=128, cache=E4)
    x.check([[some(x.rng, c, c - 300)] for c in ctx])
    x.check([[list(range(1, c))] for c in ctx])
    x.check([[list(range(64, c))] for c in ctx])
    x.check([[some(x.rng, c, c // 2)] for c in ctx])


@pytest.mark.parametrize("d,cache,n", [(128, BF, 6), (128, BF, 30), (128, E4, 12), (128, E4, 30), (64, BF, 30), (64, E4, 30)])
def test_keep_many_lists(d, cache, n):
    """From a few lists to as many as have a workgroup for whole cache lines of their rows, in place; the small
    workgroups' lists and longer ones."""
    ctx = [int(c) for c in np.random.RandomState(n).randint(1, 900, size=n)]
    for short in (False, True):
        x = Cache([1] * n, ctx, hkv=4, d=d, cache=cache)
        x.check([[some(x.rng, c, min(c, 60) if short else c - c // 5) for _ in range(4)] for c in ctx])
        x.check([[list(range(c // 3, c))[:60 if short else c] for _ in range(4)] for c in ctx])


@pytest.mark.parametrize("cache", [BF, E4])
def test_keep_into_other_pages(cache):
    """A table of fresh pages, one that begins with the old pages, and places that go on."""
    ctx, S = [100, 300, 40], 16
    x = Cache([1, 1, 1], ctx, cache=cache, spare=30)
    used = set(x.tab[x.tab >= 0].tolist())
    free = [p for p in range(x.n_blocks) if p not in used]
    to = torch.full((3, 10), -1, dtype=torch.int32)
    for s in range(3):
        to[s, :10] = torch.tensor(free[10 * s:10 * s + 10])
    lists = [[some(x.rng, c, 50) for _ in range(2)] for c in ctx]
    x.check(lists, to=to)
    to[:, 0] = x.tab[:, 0]
    x.check(lists, to=to)
    x.check([[list(range(min(c, 37))) for _ in range(2)] for c in ctx], to=to)


@pytest.mark.parametrize("cache", [BF, E4])
@pytest.mark.parametrize("per_head", [True, False])
def test_keep_paths(cache, per_head):
    """Paths of trees behind contexts of any length, with padding rows before them."""
    q_len, ctx = [5, 26, 64, 1, 0, 12, 3], [5, 90, 300, 40, 30, 8, 0]
    x = Cache(q_len, ctx, cache=cache)
    paths = []
    for s, (n, c) in enumerate(zip(q_len, ctx)):
        r0 = max(0, n - c)
        paths.append([sorted((r0 + x.rng.choice(n - r0, min(n - r0, 4), replace=False)).tolist()) if n > r0 else []
                      for _ in range(2)])
    x.check(paths, new=True, per_head=per_head)
    x.check([[[r for r in range(n - 1, n) if r >= max(0, n - c)]] * 2 for n, c in zip(q_len, ctx)], new=True, per_head=per_head)


@pytest.mark.parametrize("rows", [[3, 3], [5, 4], [0, 40], [40], [-2], [2, -1, 3], [2 ** 31 - 1], [0, 5, 0, 5, 0, 5, 0, 5] * 40])
def test_keep_bad_lists(rows):
    """Lists that do not ascend or leave the context: reported, and nothing outside the context is
    touched."""
    x = Cache([1, 1], [40, 40])
    before = [t.clone() for t in x.tensors(True)]
    r = torch.tensor([rows, [-1] * len(rows)], dtype=torch.int32, device=DEV)
    x.kv.keep(x.pages, x.tab.to(DEV), r, weights=x.w)
    refused(L.LAR_E_STATE, x.kv.sync)
    mine = torch.zeros(x.n_blocks, dtype=torch.bool)
    mine[x.tab[0].long()] = True
    for t, b in zip(x.tensors(True), before):
        assert torch.equal(t[~mine], b[~mine])


def test_lists_and_budgets_of_2_to_the_31_less_1():
    n = 2 ** 31 - 1
    x = Cache([1], [40], hkv=1)
    tab = x.tab.to(DEV)
    before = [t.clone() for t in x.tensors(True)]
    r = torch.zeros((1, 1, n), dtype=torch.int32, device=DEV)  # does not ascend, and never ends
    x.kv.keep(x.pages, tab, r, weights=x.w)
    refused(L.LAR_E_STATE, x.kv.sync)
    x.kv.plan([1], [40])
    for t, b in zip(x.tensors(True), before):
        t.copy_(b)
    r.fill_(-1)
    want = sorted(x.rng.permutation(40)[:17].tolist())
    r[0, 0, :17] = torch.tensor(want, dtype=torch.int32)
    x.kv.keep(x.pages, tab, r, weights=x.w)
    x.kv.sync()
    at = lambda j: (x.tab[0, j // 16], 0, j % 16)  # noqa: E731
    for i, j in enumerate(want):
        assert x.w[at(i)] == before[-1][at(j)]
    for c in (40, 70000):  # whole, and cut
        y = Cache([1], [c], hkv=1)
        r.fill_(7)
        y.kv.select(y.w, y.tab.to(DEV), n, rows=r)
        y.kv.sync()
        assert torch.equal(r[0, 0, :c].cpu(), torch.arange(c, dtype=torch.int32))
        for i in range(c, n, 1 << 28):
            assert bool((r[0, 0, i:i + (1 << 28)] == -1).all()), i


def test_pages_outside_the_pool_are_reported():
    for bad in (-1, 1000, 2 ** 31 - 1):
        x = Cache([1, 30], [40, 60], cache=E4)
        q = torch.randn((31, 2, 64)).to(BF).to(DEV)
        lse = torch.zeros((31, 2), dtype=torch.float32, device=DEV)
        tab = x.tab.clone()
        tab[0, 1] = tab[1, 2] = bad
        before = [t.clone() for t in x.tensors(True)]
        ok = torch.ones(x.n_blocks, dtype=torch.bool)
        ok[x.tab[x.tab >= 0].long()] = False                      # pages of no sequence
        ok[x.tab[0, 1]] = ok[x.tab[1, 2]] = True                  # and those that the table no longer names
        for call in (lambda: x.kv.weigh(x.pages, q, lse, tab.to(DEV), x.w),
                     lambda: x.kv.select(x.w, tab.to(DEV), 7),
                     lambda: x.kv.keep(x.pages, tab.to(DEV), torch.arange(3, 23, dtype=torch.int32, device=DEV).expand(2, 20).contiguous(),
                                       weights=x.w),
                     lambda: x.kv.keep(x.pages, x.tab.to(DEV), torch.arange(3, 23, dtype=torch.int32, device=DEV).expand(2, 20).contiguous(),
                                       to=tab.to(DEV), weights=x.w)):
            call()
            refused(L.LAR_E_STATE, x.kv.sync)
            for t, b in zip(x.tensors(True), before):
                assert torch.equal(t[ok], b[ok])
            x.kv.plan([1, 30], [40, 60])
            x.kv.sync()


# ------------------------------------------------------------------ far, strided, shared out
def test_past_32_bits():
    """Pages whose bytes and values lie past 2^32: a tree's attention, weights, selection, moves."""
    S, hkv, d = 16, 8, 128
    n_blocks = 2 ** 32 // (S * hkv * d) + 700
    kv = PagedKV(16, hkv, d, block_size=S, dtype=BF, cache_dtype=E4, max_seqs=2, max_tokens=300)
    pages, w = kv.new_pages(n_blocks), kv.new_weights(n_blocks)
    tab = torch.arange(n_blocks - 20, n_blocks, dtype=torch.int32, device=DEV).view(2, 10).flip(1).contiguous()
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((300, hkv, d), generator=g).to(BF) for _ in range(2))
    kv.plan([150, 150], [150, 150])
    kv.append(pages, k.to(DEV), v.to(DEV), tab)
    q = torch.randn((47, 16, d), generator=g).to(BF)
    par = [tree(7, np.random.RandomState(1)), tree(40, np.random.RandomState(2))]
    kv.plan([7, 40], [150, 150], parents=sum(par, []))
    out = kv.attend(pages, q.to(DEV), tab).cpu().double()
    held = [[R.quantise(x[150 * s:150 * s + 150], BF)[0] for x in (k, v)] for s in range(2)]
    for s, (a, n) in enumerate(((0, 7), (7, 40))):
        mask = torch.zeros((n, 150), dtype=torch.bool)
        for i, see in enumerate(seen(par[s], n, 150)[0]):
            mask[i, list(see)] = True
        want, wz, mag, big = R.attend_fast(q[a:a + n].double(), *held[s], mask, d ** -0.5)
        Batch.near(out[a:a + n], want, R.bounds(BF, mag, big, wz, d, 150, 8.0)[0], s)
    kv.plan([7, 40], [150, 150])
    lse = torch.empty((47, 16), device=DEV)
    kv.attend(pages, q.to(DEV), tab, lse=lse)
    kv.weigh(pages, q.to(DEV), lse, tab, w)
    rows = kv.select(w, tab, 60, 2, 5)
    to = torch.arange(n_blocks - 40, n_blocks - 20, dtype=torch.int32, device=DEV).view(2, 10).contiguous()
    kv.keep(pages, tab, rows, to=to, weights=w)
    kv.plan([60, 60], [60, 60])
    ko, vo = kv.read(pages, to)
    kv.sync()
    j = torch.arange(60)
    for s in range(2):
        total = 0.0
        for h in range(hkv):
            x = rows[s, h].cpu().long()
            assert (x[1:] > x[:-1]).all() and x[:2].tolist() == [0, 1] and x[-5:].tolist() == list(range(145, 150))
            for y, i in ((ko, 0), (vo, 1)):
                assert torch.equal(y[60 * s:60 * s + 60, h].cpu().double(), held[s][i][x, h])
            at = tab[s].cpu().long()
            mine = w[at[x // S].to(DEV), h, (x % S).to(DEV)]
            assert torch.equal(w[to[s].long()[j // S], h, j % S], mine)
            total += float(w[at.to(DEV), h].flatten()[:150].double().sum())
        assert abs(total / ((7, 40)[s] * 16) - 1) < 2.0 ** -16


def test_weigh_strided_queries_and_scales():
    """Queries as a slice of a fused projection, for single tokens and chunks; other scales."""
    b = Batch([1, 150, 3], [96, 300, 41], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=BF)
    fused = torch.randn((154, 12, 128)).to(BF).to(DEV)
    q = fused[:, 2:10]
    b.q = q.cpu()
    for scale in (128 ** -0.5, 0.011, 1.0):
        _, lse = b.attend(scale=scale, q=q)
        w, w2 = (b.k.new_weights(b.pages.k.shape[0]) for _ in range(2))
        b.k.weigh(b.pages, q, lse.to(DEV), b.table, w, scale=scale)
        b.k.weigh(b.pages, q.contiguous(), lse.to(DEV), b.table, w2, scale=scale)
        b.k.sync()
        assert torch.equal(w, w2)
        at = 0
        for s, (n, c) in enumerate(zip(b.q_len, b.ctx)):
            j = torch.arange(c)
            got = w.cpu()[b.table[s].cpu().long()[j // 16], :, j % 16].double()
            want, bound = weigh_ref(b, s, at, R.sees(n, c), lse[at:at + n], scale, torch.zeros(c, 2, dtype=torch.float64))
            assert ((got - want).abs() <= bound).all(), (scale, s)
            at += n


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (5, 1, 64), (64, 1, 64), (14, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5)])
def test_weigh_rows_shared_out(hq, hkv, d, window, sinks):
    """Chunks over few keys, whose rows are shared out over workgroups, heads that divide 32 and that do
    not; the same again bit for bit."""
    for q_len, ctx in (([600], [700]), ([1100, 1, 40], [1000, 200, 77])):
        b = run_weigh(q_len, ctx, hq=hq, hkv=hkv, d=d, window=window, sinks=sinks, place=False)
        _, lse = b.attend(window, sinks)
        got = []
        for _ in range(3):
            w = b.k.new_weights(b.pages.k.shape[0])
            b.k.weigh(b.pages, b.q.to(DEV), lse.to(DEV), b.table, w)
            got.append(w)
        b.k.sync()
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_select_cut_and_whole_agree():
    """Long contexts cut over workgroups and taken whole, beside short and empty ones, ties everywhere."""
    make = lambda r, s: r.randint(0, 50, s).astype(np.float32)  # noqa: E731
    check_select([70000, 0, 3, 4096, 4097, 300], 500, 4, 60, hkv=2, make=make, seed=1, q_len=[1, 0, 1, 1, 0, 0])
    check_select([262144], 1000, 0, 0, hkv=1, make=make, seed=2)
    check_select([262145], 1000, 0, 0, hkv=1, make=make, seed=3)      # more stretches than are cut
    check_select([20000] * 3, 8192, 16, 16, hkv=1, make=make, seed=4, S=128)


@pytest.mark.parametrize("c,budget,hkv", [(300001, 4096, 2), (1 << 20, 1000000, 1), ((1 << 20) + 1, 9000, 1)])
def test_select_of_many_stretches(c, budget, hkv):
    """Up to as many stretches as are cut, and one more row, with many equal weights."""
    def make(rng, shape):
        return rng.randint(0, 5000, size=shape).astype(np.float32)
    check_select([c, 9, 5000], budget, 4, 100, hkv=hkv, make=make, seed=5)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("cache", [BF, E4])
def test_drafts_are_verified_and_kept(cache):
    """Steps of drafted trees: appended, attended to, a path kept.  The cache then holds the accepted
    tokens' rows in order, as appending them alone makes it."""
    hq, hkv, d, S, steps = 8, 2, 64, 16, 6
    rng, g = np.random.RandomState(0), torch.Generator().manual_seed(0)
    kv = PagedKV(hq, hkv, d, block_size=S, dtype=BF, cache_dtype=cache, max_seqs=2, max_tokens=600)
    ref = PagedKV(hq, hkv, d, block_size=S, dtype=BF, cache_dtype=cache, max_seqs=2, max_tokens=600)
    pages, tab = kv.new_pages(60), torch.from_numpy(rng.permutation(60)[:50].reshape(2, 25).astype(np.int32)).to(DEV)
    other = ref.new_pages(60)
    ctx = [100, 37]
    draw = lambda n, h: torch.randn((n, h, d), generator=g).to(BF).to(DEV)  # noqa: E731
    k, v = draw(137, hkv), draw(137, hkv)
    for c, p in ((kv, pages), (ref, other)):
        c.plan(ctx, ctx)
        c.append(p, k, v, tab)
    for _ in range(steps):
        n = [int(rng.randint(2, 30)) for _ in ctx]
        par = [tree(m, rng) for m in n]
        kv.plan(n, [c + m for c, m in zip(ctx, n)], parents=sum(par, []))
        k, v, q = draw(sum(n), hkv), draw(sum(n), hkv), draw(sum(n), hq)
        kv.append(pages, k, v, tab)
        out = kv.attend(pages, q, tab)
        paths, start = [], np.cumsum([0] + n)
        for m, p in zip(n, par):
            a, line = int(rng.randint(m)), []
            while a >= 0:
                line.append(a)
                a = p[a]
            paths.append(line[::-1])
        most = max(map(len, paths))
        rows = torch.tensor([x + [-1] * (most - len(x)) for x in paths], dtype=torch.int32, device=DEV)
        kv.keep(pages, tab, rows, new=True)
        # the accepted tokens alone, in a cache of their own
        pick = torch.tensor([start[s] + a for s, x in enumerate(paths) for a in x], device=DEV)
        ctx = [c + len(x) for c, x in zip(ctx, paths)]
        ref.plan([len(x) for x in paths], ctx)
        ref.append(other, k[pick], v[pick], tab)
        want = ref.attend(other, q[pick], tab)
        near = (out[pick].float() - want.float()).abs() <= 2.0 ** -6 * (want.float().abs() + 1)
        assert near.all()
        kv.plan(ctx, ctx)
        ref.plan(ctx, ctx)
        for x, y in zip(kv.read(pages, tab), ref.read(other, tab)):
            assert torch.equal(bits(x), bits(y))
    kv.sync()


@pytest.mark.parametrize("cache", [BF, E4])
def test_accepted_tokens_are_weighed(cache):
    """Of a tree the accepted tokens, once in their places, with the log-sums that the tree's attention gave: as
    if they alone had been appended.  Their rows start with 0, whatever the pages' weights held there.

    The scores are the same; the two log-sums are chains of at most 150 additions in 32 bits each, with a
    logarithm of a few units at 2^-22: together off by 2 * (150 * 2^-24 + 8 * 2^-22) < 2^-14."""
    hq, hkv, d, S = 8, 2, 64, 16
    rng, g = np.random.RandomState(3), torch.Generator().manual_seed(3)
    ctx, n = [101, 30, 5], [20, 3, 40]
    par = [tree(m, rng) for m in n]
    kv = PagedKV(hq, hkv, d, block_size=S, dtype=BF, cache_dtype=cache, max_seqs=3, max_tokens=200)
    pages = kv.new_pages(30)
    tab = torch.from_numpy(rng.permutation(30)[:24].reshape(3, 8).astype(np.int32)).to(DEV)
    draw = lambda n, h: torch.randn((n, h, d), generator=g).to(BF).to(DEV)  # noqa: E731
    kv.plan(ctx, ctx)
    kv.append(pages, draw(sum(ctx), hkv), draw(sum(ctx), hkv), tab)
    k, v, q = draw(sum(n), hkv), draw(sum(n), hkv), draw(sum(n), hq)
    both = [c + m for c, m in zip(ctx, n)]
    kv.plan(n, both, parents=sum(par, []))
    kv.append(pages, k, v, tab)
    lse = torch.empty((sum(n), hq), dtype=torch.float32, device=DEV)
    kv.attend(pages, q, tab, lse=lse)
    paths, start = [], np.cumsum([0] + n)
    for m, p in zip(n, par):
        a, line = m - 1, []
        while a >= 0:
            line.append(a)
            a = p[a]
        paths.append(line[::-1])
    most = max(map(len, paths))
    kv.keep(pages, tab, torch.tensor([x + [-1] * (most - len(x)) for x in paths], dtype=torch.int32, device=DEV), new=True)
    pick = torch.tensor([start[s] + a for s, x in enumerate(paths) for a in x], device=DEV)
    now = [c + len(x) for c, x in zip(ctx, paths)]
    before = torch.full((30, hkv, S), math.nan, device=DEV)
    for s, c in enumerate(ctx):
        for j in range(c):
            before[tab[s, j // S], :, j % S] = float(j)
    got, want = before.clone(), before.clone()
    kv.plan([len(x) for x in paths], now)
    kv.weigh(pages, q[pick], lse[pick], tab, got)
    kv.append(pages, k[pick], v[pick], tab)
    own = torch.empty((len(pick), hq), dtype=torch.float32, device=DEV)
    kv.attend(pages, q[pick], tab, lse=own)
    kv.weigh(pages, q[pick], own, tab, want)
    kv.sync()
    for s, c in enumerate(now):
        for j in range(c):
            x, y = got[tab[s, j // S], :, j % S], want[tab[s, j // S], :, j % S]
            added = y - (j if j < ctx[s] else 0)
            # the sum so far, j, is rounded with what is added
            assert ((x - y).abs() <= 2.0 ** -14 * added + 2.0 ** -23 * (j + 1)).all(), (s, j)


@pytest.mark.parametrize("cache", [BF, E4])
def test_contexts_are_held_to_a_budget(cache):
    """Steps of a decoding sequence whose cache is cut when it outgrows a budget: what stays is what the
    weights of all steps say, and later tokens attend over it, head by head."""
    hq, hkv, d, S, budget, first, last = 8, 2, 64, 16, 60, 2, 9
    g = torch.Generator().manual_seed(1)
    kv = PagedKV(hq, hkv, d, block_size=S, dtype=BF, cache_dtype=cache, max_seqs=1, max_tokens=100)
    pages, tab, w = kv.new_pages(8), torch.tensor([[6, 1, 4, 0, 7, 2, 5]], dtype=torch.int32, device=DEV), kv.new_weights(8)
    held = [[torch.zeros((0, d), dtype=torch.float64) for _ in range(2)] for _ in range(hkv)]    # K, V of each head
    mine = [torch.zeros(0, dtype=torch.float64) for _ in range(hkv)]                             # their weights
    ctx, G = 0, hq // hkv
    for step, n in enumerate([50, 1, 1, 30, 1, 1, 1, 1, 25, 1]):
        ctx += n
        k, v, q = (torch.randn((n, h, d), generator=g).to(BF) for h in (hkv, hkv, hq))
        kv.plan([n], [ctx])
        kv.append(pages, k.to(DEV), v.to(DEV), tab)
        lse = torch.empty((n, hq), dtype=torch.float32, device=DEV)
        out = kv.attend(pages, q.to(DEV), tab, lse=lse).cpu().double()
        kv.weigh(pages, q.to(DEV), lse, tab, w)
        for h in range(hkv):
            for i, x in enumerate((k, v)):
                x = R.quantise(x[:, h], BF)[0] if cache == E4 else x[:, h].double()
                held[h][i] = torch.cat([held[h][i], x])
            mine[h] = torch.cat([mine[h], torch.zeros(n, dtype=torch.float64)])
            mask = R.sees(n, ctx)
            for a in range(h * G, (h + 1) * G):
                s = (q[:, a].double() @ held[h][0].T) * d ** -0.5
                p = torch.softmax(torch.where(mask, s, -math.inf), 1)
                o = p @ held[h][1]
                assert ((out[:, a] - o).abs() <= 2.0 ** -6 * (p @ held[h][1].abs())).all(), (step, a)
                mine[h] += p.sum(0)
        got = w.cpu()[tab[0].cpu().long()].transpose(0, 1).reshape(hkv, -1)[:, :ctx].double()
        for h in range(hkv):
            assert ((got[h] - mine[h]).abs() <= 2.0 ** -14 * mine[h]).all()
        rows = kv.select(w, tab, budget, first, last)
        kv.keep(pages, tab, rows, weights=w)
        kv.sync()
        for h in range(hkv):
            keep = select_ref(got[h].numpy(), budget, first, last)
            assert rows[0, h].tolist() == keep + [-1] * (budget - len(keep))
            held[h], mine[h] = [x[keep] for x in held[h]], mine[h][keep]
        ctx = min(ctx, budget)
    kv.plan([ctx], [ctx])
    for x, i in zip(kv.read(pages, tab), range(2)):
        for h in range(hkv):
            assert torch.equal(x[:, h].cpu().double(), held[h][i])


def test_captured_steps_replay():
    """Weights, selection and move, and a tree's step, in graphs on the handle's stream: replayed several
    times, with eager work between, and refused under another plan."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q_len, ctx = [12, 1, 40], [500, 300, 90]
        par = trees(q_len, ctx, 2)
        b = Trees(q_len, ctx, par, hq=8, hkv=2, d=64, S=16, dtype=BF, cache=BF, spare=40)
        q = b.q.to(DEV)
        want, _ = b.attend(lse=False)
        used = set(b.table.cpu().flatten().tolist())
        free = [p for p in range(b.pages.k.shape[0]) if p not in used][:30]
        to = torch.tensor(free, dtype=torch.int32, device=DEV).view(3, 10)
        w0 = torch.rand((b.pages.k.shape[0], 2, 16), device=DEV)
        out, w = torch.empty_like(q), w0.clone()
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=DEV)
        rows = torch.empty((3, 2, 70), dtype=torch.int32, device=DEV)

        def tree_step():
            b.k.attend(b.pages, q, b.table, out=out)

        def evict():
            b.k.attend(b.pages, q, b.table, lse=lse)
            b.k.weigh(b.pages, q, lse, b.table, w, before=w0)
            b.k.select(w, b.table, 70, 2, 5, rows=rows)
            b.k.keep(b.pages, b.table, rows, to=to, weights=w)

        for step, plan in ((tree_step, dict(parents=sum(par, []))), (evict, {})):
            b.k.plan(q_len, ctx, **plan)
            start = [t.clone() for t in b.pages.tensors()]
            step()
            b.k.sync()
            things = [out, w, rows, *[t.view(torch.uint8) for t in b.pages.tensors()]]
            eager = [t.clone() for t in things]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
            for turn in range(3):
                if step is tree_step:
                    out.fill_(3.0)
                else:
                    w.copy_(w0)
                    rows.fill_(7)
                    for t, before in zip(b.pages.tensors(), start):
                        t.copy_(before)
                graph.replay()
                b.k.sync()
                assert all(torch.equal(x, y) for x, y in zip(things, eager)), turn
                torch.randn(1000, device=DEV).sum().item()
            b.k.plan([1, 1, 1], ctx)
            keep = [t.clone() for t in things]
            graph.replay()
            refused(L.LAR_E_STATE, b.k.sync)
            assert all(torch.equal(x, y) for x, y in zip(things, keep))
        assert torch.equal(bits(out.cpu()), bits(want))


def test_calls_from_another_stream():
    """Tensors of another stream than the handle's: ordered both ways."""
    q_len, ctx = [20, 1], [900, 400]
    par = trees(q_len, ctx, 2)
    b = Trees(q_len, ctx, par, hq=8, hkv=2, d=64, S=16, dtype=BF, cache=BF, spare=20)
    want, lse = b.attend()
    b.k.plan(q_len, ctx, parents=sum(par, []))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q = b.q.to(DEV)
        x = torch.randn((4000, 4000), device=DEV)
        for _ in range(4):
            x = x @ x / 4000
        out = b.k.attend(b.pages, q + (x[0, 0] * 0).to(BF), b.table).clone()
        w = torch.rand((b.pages.k.shape[0], 2, 16), device=DEV) + x[0, 0] * 0
        rows = b.k.select(w, b.table, 50, 1, 4)
        b.k.keep(b.pages, b.table, rows.clone(), weights=w)
        w = w.cpu()
    b.k.sync()
    side.synchronize()
    assert torch.equal(bits(out.cpu()), bits(want))
    assert (rows >= 0).all()


def test_binding_refuses():
    b = Batch([3, 1], [30, 20], hq=8, hkv=2, d=64, S=16, dtype=BF, cache=BF)
    q, w = b.q.to(DEV), b.k.new_weights(b.pages.k.shape[0])
    assert (w == 0).all() and w.shape == (b.pages.k.shape[0], 2, 16)
    b.k.plan([3, 1], [30, 20])
    z = torch.zeros((4, 8), dtype=torch.float32, device=DEV)
    rows = torch.zeros((2, 2, 5), dtype=torch.int32, device=DEV)
    for call in (lambda: b.k.plan([3, 1], [30, 20], parents=[-1, 0, 0]),
                 lambda: b.k.plan([3, 1], [30, 20], parents=[-1, 0, 0, -1, 0]),
                 lambda: b.k.plan([3, 1], [30, 20], parents=[-1.0, 0.0, 0.0, -1.0]),
                 lambda: b.k.plan([3, 1], [30, 20], parents=[-1, 0, 2 ** 31, -1]),
                 lambda: b.k.weigh(b.pages, q, z.double(), b.table, w),
                 lambda: b.k.weigh(b.pages, q, z[:3], b.table, w),
                 lambda: b.k.weigh(b.pages, q, z.cpu(), b.table, w),
                 lambda: b.k.weigh(b.pages, q, z, b.table, w[:-1]),
                 lambda: b.k.weigh(b.pages, q, z, b.table, w.half()),
                 lambda: b.k.weigh(b.pages, q, z, b.table, w, before=w[:, :1]),
                 lambda: b.k.weigh(b.pages, q[:2], z, b.table, w),
                 lambda: b.k.weigh(b.pages, q, z.requires_grad_(), b.table, w),
                 lambda: b.k.weigh(b.pages, q, z.detach(), b.table, w.clone().requires_grad_()),
                 lambda: b.k.select(w, b.table[:1], 5),
                 lambda: b.k.select(w, b.table, 0),
                 lambda: b.k.select(w, b.table, 2 ** 31),
                 lambda: b.k.select(w, b.table, 2.5),
                 lambda: b.k.select(w, b.table, 5, rows=rows[:, :, :4]),
                 lambda: b.k.select(w, b.table, 5, rows=rows.long()),
                 lambda: b.k.select(w.view(-1, 1, 16), b.table, 5),
                 lambda: b.k.keep(b.pages, b.table, rows[:1]),
                 lambda: b.k.keep(b.pages, b.table, rows[:, :1]),
                 lambda: b.k.keep(b.pages, b.table, rows.long()),
                 lambda: b.k.keep(b.pages, b.table, rows.transpose(0, 1)),
                 lambda: b.k.keep(b.pages, b.table, rows.cpu()),
                 lambda: b.k.keep(b.pages, b.table, rows, weights=w[:-1]),
                 lambda: b.k.keep(b.pages, b.table, rows, to=b.table.long())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: b.k.select(w, b.table, 5, first=3, last=3), lambda: b.k.select(w, b.table, 5, first=-1),
                 lambda: b.k.plan([3, 1], [30, 20], parents=[-1, 1, 0, -1]),
                 lambda: b.k.weigh(b.pages, q, z.detach(), b.table, w, scale=0.0)):
        refused(L.LAR_E_ARG, call)
    b.k.plan([3, 1], [30, 20], parents=[-1, 0, 0, -1])
    refused(L.LAR_E_STATE, b.k.weigh, b.pages, q, z.detach(), b.table, w)
