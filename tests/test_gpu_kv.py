"""The paged key/value cache and its attention (lar_kv_*) against the definition in 64 bits."""

from __future__ import annotations

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import kv_ref as R  # noqa: E402
from gpu_util import DEV  # noqa: E402
from paper_2607_18253_amd import KvPages, LarError, PagedKV  # noqa: E402
from paper_2607_18253_amd import lar as L  # noqa: E402

BF, F16, E4 = torch.bfloat16, torch.float16, torch.float8_e4m3fn


def table_for(ctx, S, n_blocks, rng, cols=None):
    need = [-(-int(c) // S) for c in ctx]
    perm = rng.permutation(n_blocks)
    t = np.full((len(ctx), max([1] + need) if cols is None else cols), -1, np.int32)   # -1: must not be read
    at = 0
    for s, n in enumerate(need):
        t[s, :n] = perm[at:at + n]
        at += n
    return torch.from_numpy(t)


def bits(t):
    return t.contiguous().view(torch.uint8) if t.dtype == E4 else t.contiguous().view(torch.int16)


class Batch:
    """A batch with its contexts in the cache (all else in the pages is NaN) and, on the host,
    what the cache holds of each sequence in 64 bits."""

    def __init__(self, q_len, ctx, *, hq, hkv, d, S, dtype, cache, seed=0, spare=3, kv=None, edit=None,
                 max_tokens=None):
        self.q_len, self.ctx, self.d, self.dtype = list(q_len), list(ctx), d, dtype
        rng = np.random.RandomState(seed)
        g = torch.Generator().manual_seed(seed)
        n_blocks = sum(-(-c // S) for c in ctx) + spare
        self.table = table_for(ctx, S, n_blocks, rng).to(DEV)
        full = [max(0, c) for c in ctx]
        rows = [[torch.randn((c, hkv, d), generator=g).to(dtype) for _ in range(2)] for c in full]
        T = sum(q_len)
        self.q = (2.0 * torch.randn((T, hq, d), generator=g)).to(dtype)
        if edit:
            edit(self, rows)
        self.k = PagedKV(hq, hkv, d, block_size=S, dtype=dtype, cache_dtype=cache, max_seqs=max(1, len(ctx)),
                         max_tokens=max(1, T, sum(full)))
        self.pages = self.k.new_pages(n_blocks)
        for t in self.pages.tensors():
            t.view(torch.uint8).fill_(0xff)          # NaN in every type, and the largest exponent
        self.k.plan(full, full)
        if sum(full):
            self.k.append(self.pages, *(torch.cat([r[i] for r in rows]).to(DEV) for i in range(2)), self.table)
        self.held = [[R.quantise(x, dtype)[0] if cache == E4 else x.double() for x in r] for r in rows]

    def attend(self, window=0, sinks=0, scale=None, lse=True, q=None):
        self.k.plan(self.q_len, self.ctx, window=window, sinks=sinks)
        q = self.q.to(DEV) if q is None else q
        z = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV) if lse else None
        out = torch.full(q.shape, 7.0, dtype=self.dtype, device=DEV)
        self.k.attend(self.pages, q, self.table, scale=scale, out=out, lse=z)
        self.k.sync()
        return out.cpu(), None if z is None else z.cpu()

    def check(self, window=0, sinks=0, scale=None, fast=True, q=None):
        out, lse = self.attend(window, sinks, scale, q=q)
        scale = self.d ** -0.5 if scale is None else scale
        at = 0
        for s, (n, c) in enumerate(zip(self.q_len, self.ctx)):
            got, z = out[at:at + n].double(), lse[at:at + n].double()
            pad = min(n, max(0, n - c))
            assert (got[:pad] == 0).all() and (z[:pad] == -math.inf).all()
            if n > pad:
                f = R.attend_fast if fast else R.attend
                k, v = self.held[s]
                want, wz, mag, big = f(self.q[at + pad:at + n].double(), k, v, R.sees(n - pad, c, window, sinks), scale)
                bo, bz = R.bounds(self.dtype, mag, big, wz, self.d, c, float(v[torch.isfinite(v)].abs().max()))
                self.near(got[pad:], want, bo, (s, n, c))
                self.near(z[pad:], wz, bz, (s, n, c, "lse"))
            at += n

    @staticmethod
    def near(got, want, bound, what):
        fin = torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want)), what
        assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), what
        bad = ((got - want).abs() > bound) & fin
        assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / bound)[fin].max()))


# ------------------------------------------------------------------ rows into and out of pages
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hkv,d,S", [(1, 64, 1), (3, 128, 16), (8, 64, 64), (2, 128, 2)])
def test_append_and_read(dtype, e4m3, hkv, d, S):
    q_len, ctx = [1, 5, 0, 40, 3, 1], [1, 37, 9, 40, 2, 0]       # the last two with padding rows
    T, rng = sum(q_len), np.random.RandomState(3)
    n_blocks = sum(-(-c // S) for c in ctx) + 2
    tab = table_for(ctx, S, n_blocks, rng)
    kv = PagedKV(hkv, hkv, d, block_size=S, dtype=dtype, cache_dtype=E4 if e4m3 else dtype, max_seqs=6, max_tokens=T)
    pages = kv.new_pages(n_blocks)
    for t in pages.tensors():
        t.view(torch.uint8).copy_(torch.from_numpy(rng.randint(0, 256, t.view(torch.uint8).shape, np.uint8)))
    before = [t.clone() for t in pages.tensors()]
    g = torch.Generator().manual_seed(1)
    wide = [(torch.randn((T, hkv, 3 * d), generator=g) * torch.exp2(torch.randint(-20, 10, (T, hkv, 1), generator=g)
                                                                     .float())).to(dtype).to(DEV) for _ in range(2)]
    k, v = wide[0][:, :, d:2 * d], wide[1][:, :, :d]              # strided rows
    kv.plan(q_len, ctx)
    kv.append(pages, k, v, tab.to(DEV))
    ko, vo = kv.read(pages, tab.to(DEV))
    kv.sync()
    at, touched = 0, np.zeros((n_blocks, S), bool)
    for s, (n, c) in enumerate(zip(q_len, ctx)):
        for r in range(n):
            p = c - n + r
            for x, y, pool, exp in ((k, ko, pages.k, pages.k_exp), (v, vo, pages.v, pages.v_exp)):
                if p < 0:
                    assert (y[at] == 0).all()
                    continue
                page, row = int(tab[s, p // S]), p % S
                touched[page, row] = True
                if e4m3:
                    held, e = R.quantise(x[at].cpu(), dtype)
                    assert torch.equal(y[at].cpu().double(), held)
                    assert torch.equal(exp[page, :, row].cpu(), e)
                    code = R.e4m3_values()[pool[page, :, row].view(torch.uint8).cpu().numpy()]
                    assert np.array_equal(code * 2.0 ** (e.numpy().astype(float) - 127)[:, None], held.numpy())
                else:
                    assert torch.equal(bits(y[at]), bits(x[at]))
                    assert torch.equal(bits(pool[page, :, row]), bits(x[at]))
            at += 1
    rest = ~torch.from_numpy(touched).to(DEV)
    for t, b in zip(pages.tensors(), before):                     # nothing else was written
        t, b = (z.view(torch.uint8).transpose(1, 2)[rest] for z in (t, b))
        assert torch.equal(t, b)


@pytest.mark.parametrize("dtype", [BF, F16])
def test_quantise_special_rows(dtype):
    d, top = 64, float(torch.finfo(dtype).max)
    rows = [torch.zeros(d), torch.full((d,), -0.0), torch.full((d,), top), torch.full((d,), -top),
            torch.full((d,), float(torch.finfo(dtype).smallest_normal) / 4), torch.linspace(-448, 448, d),
            torch.linspace(-449, 449, d), torch.arange(d) * 2.0 ** -9, torch.arange(d) * 2.0 ** -10,
            torch.where(torch.arange(d) == 7, math.inf, torch.arange(d).float()),
            torch.where(torch.arange(d) == 9, math.nan, -torch.arange(d).float()),
            torch.full((d,), math.inf), torch.full((d,), math.nan),
            17.0 + torch.arange(d).float(), (256.0 + 16 * torch.arange(d).float()) * 3.5]
    x = torch.stack(rows).to(dtype)[:, None].contiguous()
    kv = PagedKV(1, 1, d, block_size=16, dtype=dtype, cache_dtype=E4, max_seqs=1, max_tokens=len(rows))
    pages = kv.new_pages(1)
    tab = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    kv.plan([len(rows)], [len(rows)])
    kv.append(pages, x.to(DEV), x.to(DEV), tab)
    k, v = kv.read(pages, tab)
    held, e = R.quantise(x, dtype)
    assert torch.equal(pages.k_exp[0, 0, :len(rows)].cpu(), e[:, 0])
    for y in (k, v):
        y = y.cpu().double()
        assert torch.equal(torch.isnan(y), torch.isnan(held))
        assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(held))
    assert torch.isfinite(k[:9]).all()


# ------------------------------------------------------------------ attention
HEADS = [(4, 4, 128), (8, 2, 128), (5, 1, 64), (16, 2, 64), (14, 2, 128), (32, 1, 128), (40, 1, 64), (64, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("dtype,cache", [(BF, BF), (F16, F16), (BF, E4), (F16, E4)])
def test_attend_lengths(hq, hkv, d, dtype, cache):
    """Single tokens, short and long chunks, contexts around the tiles' and pages' ends."""
    q_len = [1, 1, 1, 1, 2, 3, 1, 5, 33, 64, 70, 9, 1, 0, 1]
    ctx = [1, 31, 32, 33, 64, 65, 500, 5, 33, 200, 129, 300, 96, 50, 97]
    Batch(q_len, ctx, hq=hq, hkv=hkv, d=d, S=16, dtype=dtype, cache=cache, seed=hq).check()


@pytest.mark.parametrize("S", [1, 2, 8, 64, 1024])
@pytest.mark.parametrize("cache", [BF, E4])
def test_attend_block_sizes(S, cache):
    Batch([1, 2, 50, 1], [77, 130, 131, 1025], hq=8, hkv=2, d=128, S=S, dtype=BF, cache=cache).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (32, 0), (64, 64), (100, 4), (100, 90), (5000, 4),
                                          (33, 200)])
@pytest.mark.parametrize("cache,d", [(F16, 64), (E4, 128)])
def test_attend_window(window, sinks, cache, d):
    Batch([1, 1, 3, 80, 200, 1, 40], [1, 300, 301, 400, 200, 97, 1000], hq=8, hkv=2, d=d, S=16, dtype=F16,
          cache=cache).check(window, sinks)


@pytest.mark.parametrize("window,sinks", [(1000, 0), (1001, 1), (999, 2 ** 31 - 1), (2 ** 30 + 7, 0),
                                          (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("cache", [BF, E4])
def test_attend_window_of_whole_contexts(window, sinks, cache):
    """Windows and sinks as long as the longest context and longer, up to the largest number."""
    Batch([1, 3, 70, 40, 5], [300, 1000, 400, 1000, 3], hq=8, hkv=2, d=64, S=16, dtype=BF, cache=cache).check(window, sinks)


def test_no_plan_under_capture():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kv = PagedKV(8, 2, 64, block_size=16, max_seqs=1, max_tokens=4)
        x = torch.zeros(4, device=DEV)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            refused(L.LAR_E_STATE, kv.plan, [1], [4])
            x.fill_(1.0)
        kv.plan([1], [4])
        kv.sync()


@pytest.mark.parametrize("cache", [BF, E4])
def test_attend_padding_rows(cache):
    """Empty slots, and tokens before the first position: they see nothing."""
    for q_len, ctx in (([1, 1, 1], [0, 40, 0]), ([5, 70, 2], [3, 60, 0]), ([300, 1], [0, 0]), ([90], [1])):
        Batch(q_len, ctx, hq=8, hkv=2, d=128, S=16, dtype=BF, cache=cache).check()
        Batch(q_len, ctx, hq=8, hkv=2, d=128, S=16, dtype=BF, cache=cache).check(4, 2)


@pytest.mark.parametrize("hkv,ctx,q_len", [(1, [40000], [1]), (2, [9000, 33, 20001], [1, 1, 2]), (1, [20000], [100]),
                                           (1, [6000, 3000], [700, 30])])
@pytest.mark.parametrize("cache", [BF, E4])
def test_attend_split_contexts(hkv, ctx, q_len, cache):
    """Few rows over long contexts: the keys are split and the parts joined."""
    Batch(q_len, ctx, hq=4 * hkv, hkv=hkv, d=128, S=16, dtype=BF, cache=cache).check()


def test_attend_scores_far_apart():
    """Scores whose maximum keeps growing, rows with one key far above the others, and a scale of its own."""
    def edit(b, rows):
        for k, v in rows:
            k *= torch.linspace(0.1, 6.0, len(k))[:, None, None].to(k.dtype)
            k[len(k) // 2] *= 4
    for dtype in (BF, F16):
        Batch([1, 70, 2], [900, 600, 77], hq=8, hkv=2, d=64, S=16, dtype=dtype, cache=dtype, edit=edit).check(scale=0.5)


@pytest.mark.parametrize("q_len,G", [([3, 2], 4), ([70, 40], 4), ([300], 1), ([9], 32)])
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_attend_masked_values_have_no_part(q_len, G, dtype, bad):
    """Infinities and NaN in K and V of tokens that only later rows of the chunk see."""
    def edit(b, rows):
        for (k, v), n in zip(rows, q_len):
            v[-1, 0, 5] = bad
            v[-1, 0, 40] = -bad
            k[-1, 1 % k.shape[1], 3] = bad
            if n > 2:
                v[-n // 2, 0, 11] = bad
    b = Batch(q_len, [n + 37 for n in q_len], hq=2 * G, hkv=2, d=64, S=16, dtype=dtype, cache=dtype, edit=edit)
    out, lse = b.attend()
    at = 0
    for s, n in enumerate(q_len):
        c = b.ctx[s]
        want, wz, mag, big = R.attend(b.q[at:at + n].double(), *b.held[s], R.sees(n, c), 0.125)
        first = n - 1 if n <= 2 else n + (-n // 2)      # rows before the first bad value
        bo, bz = R.bounds(dtype, mag, big, wz, 64, c, 8.0)
        Batch.near(out[at:at + first].double(), want[:first], bo[:first], (s, "clean rows"))
        Batch.near(lse[at:at + first].double(), wz[:first], bz[:first], (s, "clean lse"))
        # a row that sees a value that is not finite is not finite where the definition is not
        got = out[at + first:at + n].double()
        assert torch.equal(torch.isfinite(got), torch.isfinite(want[first:])), s
        at += n


@pytest.mark.parametrize("n,G", [(3, 4), (2, 16), (40, 4), (9, 5)])
@pytest.mark.parametrize("cache", [BF, E4])
def test_attend_masked_values_of_split_contexts(n, G, cache):
    """NaN in V and K of the last tokens, over contexts whose keys are split: the rows before
    them stay clean through the joins, for few rows (narrow tiles) and many (wide)."""
    first = n // 2

    def edit(b, rows):
        k, v = rows[0]
        v[len(v) - n + first, 0, 5] = math.nan
        v[-1, 1, 40] = math.nan
        k[-1, 0, 3] = math.nan
    b = Batch([n], [4001], hq=2 * G, hkv=2, d=64, S=16, dtype=BF, cache=cache, edit=edit)
    out, lse = b.attend()
    k, v = (x.clone() for x in b.held[0])
    mask = R.sees(n, 4001)
    k[-1, 0], v[~torch.isfinite(v)] = 0, 0                   # for rows that do not see them
    want, wz, mag, big = R.attend_fast(b.q.double(), k, v, mask, 0.125)
    bo, bz = R.bounds(BF, mag, big, wz, 64, 4001, float(v.abs().max()))
    Batch.near(out[:first].double(), want[:first], bo[:first], "rows before the first NaN")
    Batch.near(lse[:n - 1].double(), wz[:n - 1], bz[:n - 1], "lse")
    if cache is not E4:                                      # an e4m3 row with a NaN keeps its other values
        got = out[first:n - 1, :G].double()
        assert torch.isnan(got[..., 5]).all()
        keep = [i for i in range(64) if i != 5]
        Batch.near(got[..., keep], want[first:n - 1, :G][..., keep], bo[first:n - 1, :G][..., keep], "other values")
        assert torch.isnan(out[n - 1, :G]).all() and torch.isnan(out[n - 1, G:, 40]).all()


def test_attend_repeats_bit_for_bit():
    b = Batch([1, 1, 90, 1], [3000, 20000, 5000, 4], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=BF)
    x, z = b.attend()
    for _ in range(3):
        y, w = b.attend()
        assert torch.equal(bits(x), bits(y)) and torch.equal(z, w)


def test_attend_shared_prefix_and_strided_queries():
    """Two sequences on the same first pages; queries as a slice of a fused projection."""
    b = Batch([1, 40], [96, 96], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=BF)
    b.table[1, :3] = b.table[0, :3]
    for i in range(2):
        b.held[1][i][:48] = b.held[0][i][:48]
    fused = torch.randn((41, 12, 128)).to(BF).to(DEV)
    b.q = fused[:, 2:10].cpu()
    b.check(q=fused[:, 2:10])


def test_attend_past_32_bits():
    """Pages whose bytes and values lie past 2^32."""
    S, hkv, d = 16, 8, 128
    n_blocks = 2 ** 32 // (S * hkv * d) + 700
    kv = PagedKV(16, hkv, d, block_size=S, dtype=BF, cache_dtype=E4, max_seqs=2, max_tokens=300)
    pages = kv.new_pages(n_blocks)
    tab = torch.arange(n_blocks - 20, n_blocks, dtype=torch.int32, device=DEV).view(2, 10).flip(1).contiguous()
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn((300, hkv, d), generator=g).to(BF) for _ in range(2))
    kv.plan([150, 150], [150, 150])
    kv.append(pages, k.to(DEV), v.to(DEV), tab)
    ko, vo = kv.read(pages, tab)
    assert torch.equal(ko.cpu().double(), R.quantise(k, BF)[0])
    assert torch.equal(vo.cpu().double(), R.quantise(v, BF)[0])
    q = torch.randn((41, 16, d), generator=g).to(BF)
    kv.plan([1, 40], [150, 150])
    lse = torch.empty((41, 16), device=DEV)
    out = kv.attend(pages, q.to(DEV), tab, lse=lse).cpu().double()
    kv.sync()
    for s, (a, n) in enumerate(((0, 1), (1, 40))):
        kk, vv = (x[150 * s:150 * s + 150].cpu().double() for x in (ko, vo))
        want, wz, mag, big = R.attend_fast(q[a:a + n].double(), kk, vv, R.sees(n, 150), d ** -0.5)
        bo, bz = R.bounds(BF, mag, big, wz, d, 150, 8.0)
        Batch.near(out[a:a + n], want, bo, s)


# ------------------------------------------------------------------ streams, graphs, refusals
def test_other_stream():
    b = Batch([1, 60, 2], [2000, 500, 33], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=E4)
    want, _ = b.attend()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q = b.q.to(DEV) * 1.0
        got = b.k.attend(b.pages, q, b.table).clone()
    side.synchronize()
    assert torch.equal(bits(got.cpu()), bits(want))


def test_graph_replays_on_new_values():
    """A step's append and attention captured on the handle's stream, replayed with other
    work and synchronisations between, each replay against the eager calls."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = Batch([1, 60, 2], [2000, 500, 33], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=E4)
        b.attend()
        q, out = b.q.to(DEV), torch.empty_like(b.q, device=DEV)
        k = torch.randn((63, 2, 128), device=DEV).to(BF)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.k.append(b.pages, k, k, b.table)
            b.k.attend(b.pages, q, b.table, out=out)
        seen = []
        for i in range(4):
            q.copy_(b.q.to(DEV) * (1.0 if i % 2 == 0 else 0.5))
            k.mul_(-1.5 if i else 1.0)
            out.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            b.k.append(b.pages, k, k, b.table)
            eager = b.k.attend(b.pages, q, b.table)
            torch.cuda.synchronize()
            assert torch.equal(bits(got), bits(eager)), i
            seen.append(got)
        assert not torch.equal(bits(seen[0]), bits(seen[1]))
    graph = torch.cuda.CUDAGraph()
    other = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=other):
        with pytest.raises(ValueError):
            b.k.attend(b.pages, q, b.table, out=out)
        out.fill_(1.0)
    b.k.sync()


def refused(code, f, *a, **k):
    with pytest.raises(LarError) as e:
        f(*a, **k)
    assert e.value.code == code, e.value


def test_refusals():
    ok = dict(block_size=16, max_seqs=4, max_tokens=64)
    for args, kw in (((6, 4, 128), ok), ((8, 0, 128), ok), ((8, 2, 96), ok), ((130, 2, 64), ok),
                     ((8, 2, 64), dict(ok, block_size=24)), ((8, 2, 64), dict(ok, block_size=0)),
                     ((8, 2, 64), dict(ok, max_seqs=0)), ((8, 2, 64), dict(ok, max_tokens=0)),
                     ((8, 2, 64), dict(ok, dtype=BF, cache_dtype=F16))):
        refused(L.LAR_E_ARG, PagedKV, *args, **kw)
    with pytest.raises(ValueError):
        PagedKV(8, 2, 64, dtype=torch.float32, **ok)
    kv = PagedKV(8, 2, 64, **ok)
    pages = kv.new_pages(8)
    tab = torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    q = torch.zeros((3, 8, 64), dtype=BF, device=DEV)
    new = torch.zeros((3, 2, 64), dtype=BF, device=DEV)
    refused(L.LAR_E_STATE, kv.attend, pages, q[:0], tab)            # no plan
    for a in (([1] * 5, [1] * 5), ([-1], [4]), ([1], [-1]), ([65], [65]), ([1], [1 << 30 | 1])):
        refused(L.LAR_E_ARG, kv.plan, *a)
    refused(L.LAR_E_ARG, kv.plan, [1], [4], window=-1)
    refused(L.LAR_E_ARG, kv.plan, [1], [4], window=4, sinks=-2)
    with pytest.raises(ValueError):
        kv.plan([1, 2], [4])
    kv.plan([1, 2], [32, 33])                                        # three pages needed, two columns
    refused(L.LAR_E_ARG, kv.attend, pages, q, tab)
    refused(L.LAR_E_ARG, kv.append, pages, new, new, tab)
    refused(L.LAR_E_ARG, kv.read, pages, tab)
    kv.plan([1, 2], [32, 32])
    for bad in (0.0, -1.0, math.nan, math.inf):
        refused(L.LAR_E_ARG, kv.attend, pages, q, tab, scale=bad)
    odd = torch.zeros(3 * 8 * 64 + 4, dtype=BF, device=DEV)[4:].view(3, 8, 64)
    refused(L.LAR_E_ARG, kv.attend, pages, odd, tab)                 # rows not aligned to 16 bytes
    for f, a in ((kv.attend, (pages, q[:2], tab)), (kv.attend, (pages, q.half(), tab)),
                 (kv.attend, (pages, q.cpu(), tab)), (kv.attend, (pages, q, tab.long())),
                 (kv.attend, (pages, q, tab[:1])), (kv.append, (pages, new[:, :1], new, tab)),
                 (kv.attend, (pages, q.transpose(1, 2).contiguous().transpose(1, 2), tab))):
        with pytest.raises(ValueError):
            f(*a)
    with pytest.raises(ValueError):
        kv.attend(KvPages(torch.zeros((8, 2, 32, 64), dtype=BF, device=DEV),
                          torch.zeros((8, 2, 32, 64), dtype=BF, device=DEV)), q, tab)
    with pytest.raises(ValueError):
        KvPages(pages.k.to(E4), pages.v.to(E4))
    kv.attend(pages, q, tab)                                         # and it still works
    kv.sync()
    kv.plan([], [])
    assert kv.attend(pages, q[:0], tab).shape == (0, 8, 64)
    kv.sync()


@pytest.mark.parametrize("n", [1, 50])
@pytest.mark.parametrize("page", [-1, 8, 2 ** 31 - 1])
def test_page_outside_the_pool(n, page):
    kv = PagedKV(8, 2, 64, block_size=16, max_seqs=1, max_tokens=64)
    pages = kv.new_pages(8)
    for t in pages.tensors():
        t.zero_()
    q = torch.randn((n, 8, 64), device=DEV).to(BF)
    new = torch.randn((n, 2, 64), device=DEV).to(BF)
    tab = torch.tensor([[3, page, 5, 6]], dtype=torch.int32, device=DEV)
    good = torch.tensor([[3, 4, 5, 6]], dtype=torch.int32, device=DEV)
    for call in (lambda t: kv.attend(pages, q, t), lambda t: kv.read(pages, t), lambda t: kv.append(pages, new, new, t)):
        kv.plan([n], [20 if n == 1 else 64])                         # a new token, and keys, on column 1
        call(tab)
        refused(L.LAR_E_STATE, kv.sync)
        refused(L.LAR_E_STATE, call, good)                           # sticky
        kv.plan([n], [64])                                           # a new batch
        call(good)
        kv.sync()


def test_batches_in_turn():
    """A handle's plans follow one another without waiting; each call has the plan before it."""
    b = Batch([1, 40, 2], [100, 300, 64], hq=8, hkv=2, d=128, S=16, dtype=BF, cache=BF, max_tokens=64)
    want = {}
    plans = [([1, 40, 2], [100, 300, 64]), ([1, 1, 1], [80, 300, 10]), ([30, 0, 13], [100, 300, 64]), ([1, 1, 1], [1, 0, 64])]
    for turn in range(3):
        outs = []
        for i, (n, c) in enumerate(plans):
            b.k.plan(n, c)
            outs.append((i, b.k.attend(b.pages, b.q[:sum(n)].to(DEV), b.table)))
        b.k.sync()
        for i, o in outs:
            o = bits(o.cpu())
            assert torch.equal(want.setdefault(i, o), o)
    for i, (n, c) in enumerate(plans):
        b.q_len, b.ctx = n, c
        at = 0
        out = want[i].view(BF)
        for s in range(3):
            if c[s] and n[s]:
                k, v = (x[:c[s]] for x in b.held[s])
                w, wz, mag, big = R.attend_fast(b.q[at:at + n[s]].double(), k, v, R.sees(n[s], c[s]), 128 ** -0.5)
                bo, _ = R.bounds(BF, mag, big, wz, 128, c[s], 8.0)
                Batch.near(out[at:at + n[s]].double(), w, bo, (i, s))
            at += n[s]


# ------------------------------------------------------------------ large plans, and the example
def test_attend_long_chunk_marches():
    """A chunk long enough that the workgroups of an XCD walk over the same keys: 32 tiles of
    1094 key tiles and one of 1; the reference in 64 bits on the GPU, row by block of rows."""
    hq, hkv, d, S, n, c = 4, 1, 64, 16, 2049, 70017
    kv = PagedKV(hq, hkv, d, block_size=S, max_seqs=1, max_tokens=c)
    g = torch.Generator(device=DEV).manual_seed(4)
    k, v = (torch.randn((c, hkv, d), device=DEV, generator=g).to(BF) for _ in range(2))
    q = (2 * torch.randn((n, hq, d), device=DEV, generator=g)).to(BF)
    blocks = -(-c // S)
    tab = torch.randperm(blocks, device=DEV, generator=g).int()[None].contiguous()
    pages = kv.new_pages(blocks)
    kv.plan([c], [c])
    kv.append(pages, k, v, tab)
    kv.plan([n], [c])
    lse = torch.empty((n, hq), device=DEV)
    out = kv.attend(pages, q, tab, lse=lse)
    kv.sync()
    kk, vv = k[:, 0].double(), v[:, 0].double()
    for h in range(hq):
        for a in range(0, n, 512):
            b = min(n, a + 512)
            mask = R.sees(b - a, c - n + b).to(DEV)
            m = mask.shape[1]
            want, wz, mag, big = R.attend_fast(q[a:b, h:h + 1].double(), kk[:m, None], vv[:m, None], mask, d ** -0.5)
            bo, bz = R.bounds(BF, mag, big, wz, d, c, 6.0)
            Batch.near(out[a:b, h:h + 1].double(), want.to(DEV), bo.to(DEV), (h, a))
            Batch.near(lse[a:b, h:h + 1].double(), wz.to(DEV), bz.to(DEV), (h, a, "lse"))


@pytest.mark.parametrize("seed", range(12))
def test_attend_random_batches(seed):
    """Random mixed batches: single tokens, short and long chunks, padding, windows, types."""
    r = np.random.RandomState(100 + seed)
    hkv = int(r.choice([1, 2, 3]))
    G, d = int(r.choice([1, 3, 4, 8, 16])), int(r.choice([64, 128]))
    dtype = [BF, F16][r.randint(2)]
    cache = [dtype, E4][r.randint(2)]
    n_seq = r.randint(1, 14)
    q_len = [int(x) for x in np.where(r.rand(n_seq) < 0.5, 1, np.exp(r.uniform(0, 5.2, n_seq)))]
    ctx = [int(x) for x in np.exp(r.uniform(0, 7.6, n_seq))]
    ctx = [c if r.rand() < 0.15 else c + n for c, n in zip(ctx, q_len)]
    window, sinks = (0, 0) if r.rand() < 0.5 else (int(np.exp(r.uniform(0, 6))), int(r.choice([0, 1, 4, 50])))
    Batch(q_len, ctx, hq=hkv * G, hkv=hkv, d=d, S=int(r.choice([4, 16, 16, 32, 128])), dtype=dtype, cache=cache,
          seed=seed).check(window, sinks)


def test_calibration_runs_the_batches():
    """The example: batches of a small instance through append and attention, its
    coefficients fitted and handed to the simulation."""
    from paper_2607_18253_amd import calibrate as K
    inst = K.Instance(n_q_heads=8, n_kv_heads=2, head_dim=64, layers=2, token_budget=256, max_seqs=24, chunk_cap=64,
                      kv_blocks=600, max_ctx=512)
    some = K.batches(inst, 9, seed=2)
    ms = K.measure(inst, some, e4m3=True)
    assert ms.shape == (9,) and np.isfinite(ms).all() and (ms > 0).all()
    c = K.fit([b.features() for b in some], ms)
    assert np.isfinite(c).all() and (c >= 0).all() and c.any()
    assert (K.main(["--layers", "2", "--kv-blocks", "2000", "--max-seqs", "32", "--token-budget", "512", "--max-ctx",
                    "2048", "--chunk-cap", "128", "--batches", "12"]) >= 0).all()
