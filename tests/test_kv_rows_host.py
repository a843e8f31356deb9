"""The host side of trees, weights, selections and moves on the paged cache, on a stand-in for the
HIP runtime: what a plan with trees hands to the kernels, and which calls are refused.  No GPU."""

from __future__ import annotations

import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2607_18253_amd.kv import KvConfig, KvPagesArg, KvRowsArg
from test_kv_calls_host import Tensor, binding  # noqa: F401  (the fixture)

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2607_18253_amd", "csrc")
E_ARG, E_CAPACITY, E_STATE = -1, -3, -2


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    out = str(tmp_path_factory.mktemp("kv") / "libkvrows.so")
    stub = os.path.join(HERE, "hip_stub")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", stub, os.path.join(CSRC, "kv_api.cpp"),
                    os.path.join(CSRC, "kv_rows_api.cpp"), os.path.join(stub, "kv_rows_host.cpp"), "-o", out], check=True)
    L = C.CDLL(out)
    vp, i32 = C.c_void_p, C.c_int32
    L.lar_kv_plan.argtypes = [vp, i32, vp, vp, i32, i32]
    L.lar_kv_plan_tree.argtypes = [vp, i32, vp, vp, vp, i32, i32]
    L.lar_kv_attend.argtypes = [vp, vp, vp, vp, i32, C.c_double, vp, vp]
    L.lar_kv_weigh.argtypes = [vp, vp, vp, vp, i32, C.c_double, vp, vp, vp]
    L.lar_kv_select.argtypes = [vp, vp, C.c_int64, vp, i32, i32, i32, i32, vp]
    L.lar_kv_keep.argtypes = [vp, vp, vp, i32, vp, i32, vp, i32, i32, i32, vp]
    L.lar_kv_destroy.argtypes = [vp]
    L.lar_kv_create.argtypes = [C.POINTER(vp), vp]
    L.lar_kv_error_string.argtypes, L.lar_kv_error_string.restype = [vp], C.c_char_p
    return L


class Handle:
    """A handle, pages and rows that no kernel looks at."""

    def __init__(self, lib, max_seqs=8, max_tokens=256, hq=8, hkv=2, d=64, S=16):
        self.L, self.h, self.hkv = lib, C.c_void_p(), hkv
        cfg = KvConfig(hq, hkv, d, 1, 1, S, max_seqs, max_tokens, 0, None)
        assert lib.lar_kv_create(C.byref(self.h), C.byref(cfg)) == 0
        self.pages, self.q = KvPagesArg(4096, 8192, None, None, 64), KvRowsArg(4096, hq * d, d)

    def plan(self, q_len, ctx, parents=None, window=0, sinks=0):
        q, c = np.array(q_len, np.int32), np.array(ctx, np.int32)
        if parents is None:
            return self.L.lar_kv_plan(self.h, len(q), q.ctypes.data, c.ctypes.data, window, sinks)
        up = np.array(parents, np.int32)
        return self.L.lar_kv_plan_tree(self.h, len(q), q.ctypes.data, c.ctypes.data, up.ctypes.data, window, sinks)

    def attend(self):
        return self.L.lar_kv_attend(self.h, C.byref(self.pages), C.byref(self.q), 4096, 1 << 20, 0.125, 4096, None)

    def weigh(self, cols=1 << 20, scale=0.125, lse=4096, before=1 << 30, weights=1 << 30, q=None):
        return self.L.lar_kv_weigh(self.h, C.byref(self.pages), C.byref(self.q if q is None else q), 4096, cols, scale,
                                   lse, before, weights)

    def select(self, budget=4, first=0, last=0, weights=4096, n_blocks=64, cols=1 << 20, rows=4096, table=4096):
        return self.L.lar_kv_select(self.h, weights, n_blocks, table, cols, budget, first, last, rows)

    def keep(self, cols=1 << 20, to=None, to_cols=0, rows=4096, n_rows=4, per_head=1, fresh=0, weights=None):
        return self.L.lar_kv_keep(self.h, C.byref(self.pages), 4096, cols, to, to_cols, rows, n_rows, per_head, fresh,
                                  weights)

    def numbers(self, f, what, room):
        got = np.empty(room, np.int32)
        n = f(what, got.ctypes.data_as(C.c_void_p), room)
        assert n <= room
        return got[:n].copy()

    def trees(self, what, room):
        return self.numbers(self.L.stub_trees, what, room)

    def arrays(self, what):
        return self.numbers(self.L.stub_plan, what, 1 << 20)

    def close(self):
        self.L.lar_kv_destroy(self.h)


def tree(n, rng, spread=4, roots=1):
    return [-1 if i < roots else int(rng.randint(max(0, i - spread), i)) for i in range(n)]


def seen(par, n, c, window=0, sinks=0):
    """Keys that each new token sees, and its place, by walking up."""
    base, r0 = c - n, max(0, n - c)
    out, places = [], []
    for i in range(n):
        if i < r0:
            out.append(set())
            places.append(-1)
            continue
        line, a = [], i
        while a >= 0:
            line.append(a)
            a = par[a]
        line = line[::-1]
        keys = list(range(max(0, base))) + [base + a for a in line]
        here = len(keys) - 1
        out.append({k for p, k in enumerate(keys) if not window or p > here - window or p < sinks})
        places.append(here)
    return out, places


@pytest.mark.parametrize("seed", range(24))
def test_stretches_of_trees_hold_what_each_token_sees(lib, seed):
    """Every visible key of every row is in one stretch of the row's tile, records say which ones
    they are, parts of a tile are in slots of their own and all joined, and places are in range."""
    rng = np.random.RandomState(seed)
    hkv, G = int(rng.choice([1, 2, 8])), int(rng.choice([1, 4, 5, 8, 64]))
    S = int(rng.choice([1, 16, 64]))
    q_len, ctx, par = [], [], []
    for _ in range(int(rng.randint(1, 7))):
        n = int(rng.choice([1, 2, 3, 9, 33, 64, 130, 300]))
        c = int(rng.choice([0, n - 1, n, n + 1, n + 37, n + 64, n + 700, n + 5000]))
        kind = rng.randint(3)
        r0 = max(0, n - c)
        p = list(range(-1, n - 1)) if kind == 0 else tree(n, rng, int(rng.choice([1, 3, 500])))
        p = [-1 if i == r0 or (x < r0 and i > r0) else x for i, x in enumerate(p)]
        q_len.append(n), ctx.append(c), par.append(p)
    window, sinks = (int(rng.choice([1, 3, 40, 600])), int(rng.choice([0, 1, 70]))) if seed % 2 else (0, 0)
    x = Handle(lib, max_seqs=len(q_len), max_tokens=sum(q_len), hq=hkv * G, hkv=hkv, S=S)
    assert x.plan(q_len, ctx, sum(par, []), window, sinks) == 0, lib.lar_kv_error_string(x.h)
    assert x.attend() == 0
    spans = x.trees(0, 7 * len(q_len)).reshape(-1, 7)
    segs = [(K, g) for what, K in ((1, 32), (2, 64)) for g in x.arrays(what).reshape(-1, 10)]
    joins = x.arrays(5).reshape(-1, 8)
    eff = window if window < max(c for c, n in zip(ctx, q_len) if n) else 0
    room = int(sum(n * (w + 1) for n, (*_, t, w, _, _) in zip(q_len, spans) if t >= 0))
    words = x.trees(1, room).view(np.uint32)
    assert (len(words) > 0) == (room > 0)
    slots, parts, q0 = set(), {}, 0
    for s, (n, c, p) in enumerate(zip(q_len, ctx, par)):
        assert tuple(spans[s][:3]) == (q0, n, c)
        chain = p[max(0, n - c):] == [-1] + list(range(max(0, n - c), n - 1)) if c else True
        assert (spans[s][3] < 0) == chain
        mine = [(K, g) for K, g in segs if g[4] == s]
        if chain:
            q0 += n
            continue
        assert len({K for K, _ in mine}) == 1
        keys, places = seen(p, n, c, eff, sinks if eff else 0)
        base, block, w = c - n, max(0, c - n) >> 5, int(spans[s][4])
        for i in range(n):
            rec = words[spans[s][3] + i * (w + 1):][:w + 1]
            bits = {32 * (block + b // 32) + b % 32 for b in range(32 * w) if rec[1 + b // 32] >> (b % 32) & 1}
            assert bits == {k for k in keys[i] if k >= 32 * block}
            if i >= max(0, -base):
                assert rec[0] == places[i]
        for h in range(hkv):
            cover = [[] for _ in range(n)]
            for K, g in (x for x in mine if x[1][3] == h):
                rows, t0tok = 32 if K == 32 else 256, g[0]
                t0tok, ntok, p0, _, _, ns, fw, t0, t1, slot = g
                assert p0 == base + (t0tok - q0) and 0 < ntok * G <= rows and 0 <= t0 <= t1
                for t in range(t0, t1):
                    kb = (t if t < ns else fw + t - ns) * K
                    assert 0 <= kb <= p0 + ntok - 1
                    for i in range(t0tok - q0, t0tok - q0 + ntok):
                        cover[i].append(kb)
                key = (K, s, h, t0tok)
                parts.setdefault(key, []).append((int(t0), int(t1), int(slot)))
            for i in range(n):
                assert len(set(cover[i])) == len(cover[i])
                got = set(cover[i])
                assert all(k // K * K in got for k in keys[i])   # K: all of a sequence's tiles are of one kind
        q0 += n
    want = {}
    for key, p in parts.items():
        if len(p) == 1:
            assert p[0][2] == -1
            continue
        p.sort()
        assert all(a[1] == b[0] for a, b in zip(p, p[1:]))
        ids = [a[2] for a in p]
        assert ids == list(range(ids[0], ids[0] + len(ids)))
        mine = {(key[0], i) for i in ids}
        assert not slots & mine
        slots |= mine
        want[key] = (ids[0], len(ids))
    got = {}
    for q0_, ntok, p0, head, slot, n, row0, wide in joins:
        s = next(i for i, sp in enumerate(spans) if sp[0] <= q0_ < sp[0] + sp[1])
        if spans[s][3] >= 0:
            got[(64 if wide else 32, s, head, q0_)] = (slot, n)
    assert got == want
    x.close()


def test_chains_are_ordinary_batches(lib):
    """Parents that follow one another make the plan that lengths alone make, whatever padding rows
    have for parents; another tree is another plan."""
    x = Handle(lib)
    lib.stub_attend_plan.restype = C.c_uint64
    ids = []
    for parents in (None, [-1, 0, 1, 2, -1, 7, 0, -1, 1], [-1, 0, 1, 2, -1, 7, 9, -1, 1]):
        q = [4, 1, 4] if parents is None else [4, 1, 4]
        if parents is not None:
            parents = parents[:5] + [99, 98, -1, 2]
        assert x.plan(q, [50, 9, 2], parents) == 0, lib.lar_kv_error_string(x.h)
        assert x.attend() == 0 and len(x.trees(1, 1)) == 0
        ids.append(lib.stub_attend_plan())
    assert len(set(ids)) == 1
    for parents in ([-1, 0, 0, 2], [-1, 0, 1, 1], [-1, 0, 0, 1], [-1, -1, -1, -1]):
        assert x.plan([4], [50], parents) == 0
        assert x.attend() == 0 and len(x.trees(1, 1)) > 0
        ids.append(lib.stub_attend_plan())
    assert len(set(ids)) == 5
    x.close()


def test_padding_rows_have_no_part_in_a_trees_plan(lib):
    """Their parents are not looked at: a captured call may be replayed under the same trees whatever they are."""
    x = Handle(lib)
    lib.stub_attend_plan.restype = C.c_uint64
    ids, words = [], []
    for pad in ([-1, -1], [99, -7], [1, 0]):
        assert x.plan([3, 5], [50, 3], [-1, 0, 0] + pad + [-1, 2, 2]) == 0, lib.lar_kv_error_string(x.h)
        assert x.attend() == 0
        ids.append(lib.stub_attend_plan())
        words.append(x.trees(1, 3 * 2 + 5 * 2).tolist())
    assert len(set(ids)) == 1 and words[0] == words[1] == words[2]
    assert x.plan([3, 5], [50, 3], [-1, 0, 0, -1, -1, -1, 2, -1]) == 0 and x.attend() == 0
    assert lib.stub_attend_plan() not in ids
    x.close()


def test_bad_trees_are_refused(lib):
    x = Handle(lib, max_tokens=40000, max_seqs=64)
    ok = [-1, 0, 0]
    assert x.plan([3], [9], ok) == 0
    for parents in ([0, 0, 0], [-1, 1, 0], [-1, 2, 0], [-1, 0, -2], [-1, 0, 2 ** 31 - 1], [-1, -2 ** 31, 0]):
        assert x.plan([3], [9], parents) == E_ARG, parents
    assert x.plan([3], [1], [5, 5, -1]) == 0            # two padding rows
    assert x.plan([3], [2], [5, 0, 1]) == E_ARG         # a parent that is one
    assert x.plan([1024], [2000], [-1, 0, 0] + list(range(2, 1023))) == 0
    assert x.plan([1025], [2000], [-1, 0, 0] + list(range(2, 1024))) == E_ARG
    assert x.plan([20000], [30000], list(range(-1, 19999))) == 0   # a chain has no such limit
    par = [-1, 0, 0] + list(range(2, 1023))
    assert x.plan([1024] * 16, [2000] * 16, par * 16) == 0
    assert x.plan([1024] * 16 + [3], [2000] * 17, par * 16 + ok) == E_CAPACITY
    assert lib.lar_kv_plan_tree(x.h, 1, None, None, None, 0, 0) == E_ARG
    x.close()


def test_rows_calls_check_their_arguments(lib):
    x = Handle(lib)
    got = np.zeros(4, np.int32)
    g = got.ctypes.data_as(C.c_void_p)
    for call in (x.weigh, x.select, x.keep):
        assert call() == E_STATE                        # no plan
    assert x.plan([1, 20, 0], [40, 100, 300]) == 0
    assert x.weigh() == 0 and lib.stub_weigh(g) == 1
    assert tuple(got[:3]) == (1, 3, got[2]) and got[2] > 0   # 100 keys of the chunk: one block
    for bad in (dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(lse=None), dict(before=None),
                dict(weights=None), dict(cols=6), dict(before=(1 << 30) + 16), dict(before=(1 << 30) - 16),
                dict(q=KvRowsArg(4100, 512, 64)), dict(q=KvRowsArg(4096, 513, 64))):
        assert x.weigh(**bad) == E_ARG and lib.stub_weigh(g) == 0, bad
    size = 64 * 2 * 16 * 4                              # of the weights: right beside is apart
    assert x.weigh(before=(1 << 30) + size) == 0 and x.weigh(before=(1 << 30) - size) == 0
    assert x.weigh(cols=7) == 0                         # the sequence without new tokens is not looked at
    assert x.select(cols=19) == 0 and x.keep(cols=19) == 0
    for bad in (dict(budget=0), dict(budget=-1), dict(first=5), dict(last=5), dict(first=2, last=3), dict(first=-1),
                dict(last=-1), dict(first=2 ** 31 - 1, last=2 ** 31 - 1), dict(weights=None), dict(rows=None),
                dict(table=None), dict(cols=18), dict(n_blocks=0), dict(n_blocks=2 ** 31)):
        assert x.select(**bad) == E_ARG, bad
    assert x.keep() == 0 and lib.stub_keep(g) == 1 and tuple(got) == (2, 4, 0, 1)
    assert x.keep(to=8192, to_cols=1, n_rows=16, per_head=0) == 0 and lib.stub_keep(g) == 1
    assert tuple(got) == (1, 16, 0, 0)
    for bad in (dict(rows=None), dict(n_rows=-1), dict(per_head=2), dict(fresh=3), dict(cols=18),
                dict(to=8192, to_cols=1, n_rows=17), dict(to=8192, to_cols=18, fresh=1)):
        assert x.keep(**bad) == E_ARG and lib.stub_keep(g) == 0, bad
    assert x.keep(n_rows=0) == 0 and lib.stub_keep(g) == 0
    assert x.plan([3], [9], [-1, 0, 0]) == 0
    assert x.weigh() == E_STATE and x.select() == 0 and x.keep(fresh=1) == 0
    assert x.plan([], []) == 0                          # nothing to do
    lib.stub_weigh(g), lib.stub_keep(g)
    assert x.weigh() == 0 and x.select() == 0 and x.keep() == 0
    assert lib.stub_weigh(g) == 0 and lib.stub_keep(g) == 0
    x.close()


def test_weights_have_the_key_blocks_that_are_seen(lib):
    """Chunks under a window: blocks of 256 keys with one that some token sees, no others, and of each the
    tokens that see one of it."""
    rng, got = np.random.RandomState(0), np.zeros(3, np.int32)
    g = got.ctypes.data_as(C.c_void_p)
    for _ in range(400):
        n = int(rng.randint(1, 1200))
        c = max(0, n + int(rng.choice([-n, -7, 0, 1, 255, 256, 257, 900, 4000])))
        window, sinks = int(rng.choice([0, 1, 2, 255, 256, 257, 600, 5000])), int(rng.choice([0, 1, 256, 300, 2 ** 31 - 1]))
        p = np.arange(c - n, c)[:, None]
        j = np.arange(c)[None]
        mask = (j <= p) & ((window == 0) | (j > p - window) | (j < sinks))
        want = [kb for kb in range(0, c, 256) if mask[:, kb:kb + 256].any()]
        assert lib.stub_seen_blocks(c, n, window, sinks, 0, g) == len(want)
        for i, kb in enumerate(want):
            lib.stub_seen_blocks(c, n, window, sinks, i, g)
            t = np.flatnonzero(mask[:, kb:kb + 256].any(1))
            assert got[0] == kb and got[1] == t[0] and t[-1] < got[2] <= n, (c, n, window, sinks, kb)
            # a last block ends with the context: its tokens are counted as if it went on
            assert got[2] == t[-1] + 1 or kb + 256 > c, (c, n, window, sinks, kb)
    x = Handle(lib, max_seqs=4, max_tokens=4096)
    assert x.plan([512, 1, 40], [100000, 5000, 90], window=4096, sinks=4) == 0 and x.weigh() == 0
    lib.stub_weigh(g)
    first = (100000 - 512 - 4095) // 256
    assert got[0] == 1 + (391 - first) + 1
    x.close()


@pytest.mark.parametrize("ctx", [1 << 26, (1 << 29) + 77, 1 << 30])
def test_rows_of_far_key_blocks_are_counted_in_32_bits(lib, ctx):
    """64 heads for a kv head and a chunk far from the sinks: the tokens of every block are within the chunk."""
    got = np.zeros(3, np.int32)
    for n, window, sinks in ((40, 300, 5), (5000, 4096, 0), (1 << 24, 1, 1000), (1, 1 << 20, 0)):
        for i in range(lib.stub_seen_blocks(ctx, n, window, sinks, 0, got.ctypes.data_as(C.c_void_p))):
            lib.stub_seen_blocks(ctx, n, window, sinks, i, got.ctypes.data_as(C.c_void_p))
            kb, t0, t1 = (int(x) for x in got)
            assert 0 <= kb < ctx and 0 <= t0 < t1 <= n and t1 * 64 < 2 ** 31
            if i > 64:
                break
        assert x_blocks(lib, ctx, n, window, sinks) == lib.stub_seen_blocks(ctx, n, window, sinks, 0, got.ctypes.data_as(C.c_void_p))


def x_blocks(lib, ctx, n, window, sinks):
    """Blocks of one chunk that a call hands on."""
    got = np.zeros(4, np.int32)
    x = Handle(lib, max_seqs=1, max_tokens=n, hq=64, hkv=1, S=65536)
    assert x.plan([n], [ctx], window=window, sinks=sinks) == 0 and x.weigh() == 0
    lib.stub_weigh(got.ctypes.data_as(C.c_void_p))
    x.close()
    return int(got[0])


def test_long_chunks_of_many_heads_are_refused(lib):
    """Rows of a sequence are counted in 32 bits."""
    x = Handle(lib, max_seqs=1, max_tokens=1 << 24, hq=64, hkv=1)
    assert x.plan([1 << 24], [1 << 24]) == 0 and x.weigh(cols=1 << 21) == 0
    x.close()
    x = Handle(lib, max_seqs=1, max_tokens=(1 << 24) + 1, hq=64, hkv=1)
    assert x.plan([(1 << 24) + 1], [(1 << 24) + 1]) == 0 and x.weigh(cols=1 << 21) == E_CAPACITY
    x.close()


def test_launches_of_too_many_threads_are_refused(lib):
    """A launch has less than 2^32 threads: the last batch that fits, and one more sequence.  No call counts
    workgroups that it does not launch."""
    most = 1 << 20
    x = Handle(lib, max_seqs=most, max_tokens=1, hkv=8)

    def plan(n, ctx, first=1, window=0):
        assert x.plan([1] + [0] * (n - 1), [first] + [ctx] * (n - 1), window=window) == 0

    plan((1 << 18) - 1, 5)
    assert x.keep(n_rows=4096) == 0                    # 8 heads, K and V: 16 workgroups of 1024
    assert x.keep(n_rows=4096, weights=4096) == E_CAPACITY
    plan(1 << 18, 5)
    assert x.keep(n_rows=4096) == E_CAPACITY
    assert b"1024 threads" in lib.lar_kv_error_string(x.h)
    plan(most - 1, 5)
    assert x.keep(n_rows=4) == 0                       # of 256
    plan(most, 5)
    assert x.keep(n_rows=4) == E_CAPACITY
    assert x.select() == 0                             # 8 heads: 8 workgroups of 256
    plan(most - 1, 5, first=2049)
    assert x.select() == 0                             # of 512
    plan(most, 5, first=2049)
    assert x.select() == E_CAPACITY
    x.close()
    x = Handle(lib, max_seqs=most, max_tokens=1, hq=16, hkv=16)
    plan(most - 1, 5, first=100, window=7)
    assert x.weigh() == 0 and x.weigh(before=1 << 40) == 0
    plan(most, 5, first=100, window=7)
    assert x.weigh() == 0                              # in place nothing is carried over
    assert x.weigh(before=1 << 40) == E_CAPACITY
    assert x.select() == E_CAPACITY
    plan(most, 5, first=100)
    assert x.weigh(before=1 << 40) == 0                # without a window neither
    x.close()


@pytest.mark.parametrize("current", [0, 1])
def test_calls_go_to_the_handles_device(lib, current):
    """A handle made on device 1 works on it whichever device is current, and leaves that one current."""
    lib.stub_use(1)
    x = Handle(lib)
    lib.stub_use(current)
    lib.stub_calls(0)
    for call in (lambda: x.plan([1, 5], [40, 100]), x.weigh, x.select, x.keep,
                 lambda: x.plan([3], [100], [-1, 0, 0]), x.attend, lambda: x.keep(fresh=1)):
        lib.stub_calls(1)
        assert call() == 0
        assert lib.stub_device() == current
        assert lib.stub_calls(0) == 0 and lib.stub_calls(1) > 0
    x.close()
    lib.stub_use(0)


def test_launches_carry_their_plan(lib):
    lib.stub_device_plan.restype = lib.stub_rows_plan.restype = C.c_uint64
    x = Handle(lib)
    ids = set()
    for i, (call, plan) in enumerate(((x.weigh, {}), (x.select, {}), (x.keep, {}), (lambda: x.keep(fresh=1), dict(parents=[-1, 0, 0])))):
        assert x.plan([3], [50 + i], **plan) == 0 and x.attend() == 0 and call() == 0
        assert lib.stub_rows_plan(min(i, 2)) == lib.stub_device_plan()
        ids.add(lib.stub_device_plan())
    assert len(ids) == 4
    # a batch without new tokens is a plan too
    assert x.plan([0, 0], [50, 60]) == 0 and x.select() == 0 and lib.stub_rows_plan(1) not in ids
    x.close()


def test_plans_without_new_tokens_reach_the_device(lib):
    x = Handle(lib)
    assert x.plan([3], [50]) == 0 and x.attend() == 0
    lib.stub_device_plan.restype = lib.stub_rows_plan.restype = C.c_uint64
    before = lib.stub_device_plan()
    assert x.plan([0], [50]) == 0 and x.keep() == 0
    assert lib.stub_device_plan() == lib.stub_rows_plan(2) != before
    x.close()


# ------------------------------------------------------------------ the binding's checks
def test_tensors_of_another_device_are_refused(binding):  # noqa: F811
    import torch
    from paper_2607_18253_amd import KvPages
    B, F, I = torch.bfloat16, torch.float32, torch.int32
    pages = KvPages(*(Tensor((9, 2, 16, 64), B) for _ in range(2)))
    q, tab, lse, w = Tensor((3, 8, 64), B), Tensor((1, 4), I), Tensor((3, 8), F), Tensor((9, 2, 16), F)
    rows = Tensor((1, 2, 5), I)
    binding.weigh(pages, q, lse, tab, w, before=Tensor((9, 2, 16), F, at=1 << 20))
    binding.select(w, tab, 5, rows=rows)
    binding.keep(pages, tab, rows, to=tab, weights=w)
    binding.keep(pages, tab, Tensor((1, 5), I), new=True)
    assert [n for n, _ in binding._L.calls] == ["lar_kv_weigh", "lar_kv_select", "lar_kv_keep", "lar_kv_keep"]
    far = lambda t: Tensor(t.shape, t.dtype, device=1)  # noqa: E731
    for call in (lambda: binding.weigh(pages, far(q), lse, tab, w), lambda: binding.weigh(pages, q, far(lse), tab, w),
                 lambda: binding.weigh(pages, q, lse, far(tab), w), lambda: binding.weigh(pages, q, lse, tab, far(w)),
                 lambda: binding.weigh(pages, q, lse, tab, w, before=far(w)), lambda: binding.select(far(w), tab, 5, rows=rows),
                 lambda: binding.select(w, far(tab), 5, rows=rows), lambda: binding.select(w, tab, 5, rows=far(rows)),
                 lambda: binding.keep(pages, far(tab), rows), lambda: binding.keep(pages, tab, far(rows)),
                 lambda: binding.keep(pages, tab, rows, to=far(tab)), lambda: binding.keep(pages, tab, rows, weights=far(w))):
        with pytest.raises(ValueError, match="cuda:0"):
            call()
    assert len(binding._L.calls) == 4
    name, args = binding._L.calls[2]
    assert args[4] == tab.at and args[7:10] == (5, 1, 0)
    name, args = binding._L.calls[3]
    assert args[4] is None and args[7:10] == (5, 0, 1) and args[10] is None


def test_shapes_are_refused(binding):  # noqa: F811
    import torch
    from paper_2607_18253_amd import KvPages
    B, F, I = torch.bfloat16, torch.float32, torch.int32
    pages = KvPages(*(Tensor((9, 2, 16, 64), B) for _ in range(2)))
    q, tab, lse, w = Tensor((3, 8, 64), B), Tensor((1, 4), I), Tensor((3, 8), F), Tensor((9, 2, 16), F)
    for call in (lambda: binding.weigh(pages, Tensor((2, 8, 64), B), lse, tab, w),
                 lambda: binding.weigh(pages, q, Tensor((3, 7), F), tab, w),
                 lambda: binding.weigh(pages, q, lse, tab, Tensor((8, 2, 16), F)),
                 lambda: binding.weigh(pages, q, lse, tab, Tensor((9, 16, 2), F)),
                 lambda: binding.weigh(pages, q, lse, tab, w, before=Tensor((10, 2, 16), F)),
                 lambda: binding.weigh(pages, q, lse, Tensor((0, 4), I), w),
                 lambda: binding.select(Tensor((9, 2, 8), F), tab, 5),
                 lambda: binding.select(w, tab, 5, rows=Tensor((2, 2, 5), I)),
                 lambda: binding.select(w, tab, 0), lambda: binding.select(w, tab, -5),
                 lambda: binding.keep(pages, tab, Tensor((1, 3, 5), I)), lambda: binding.keep(pages, tab, Tensor((2, 5), I)),
                 lambda: binding.keep(pages, tab, Tensor((5,), I)), lambda: binding.keep(pages, tab, Tensor((1, 2, 5), torch.int64)),
                 lambda: binding.keep(pages, tab, Tensor((1, 2, 5), I), weights=Tensor((8, 2, 16), F))):
        with pytest.raises(ValueError):
            call()
    assert not binding._L.calls


def test_parents_are_not_cut(binding):  # noqa: F811
    for bad in ([-1, 0], [-1, 0, 0, 0], [-1, 0, 0.5], [-1, 0, 2 ** 31], [[-1, 0, 0]], 3):
        with pytest.raises(ValueError):
            binding.plan([3], [50], parents=bad)
    assert not binding._L.calls
    binding.plan([3], [50], parents=(-1, 0, 0))
    assert binding._L.calls[0][0] == "lar_kv_plan_tree"
