"""Batch-time coefficients of the attention, measured on the GPU that serves.

The simulation times a token batch by T = a + b*P + c*D + d*C + e*A (lar_instance_params):
P prefill tokens, D decoding sequences, C their context (KV-cache reads), A the prefill
chunks' attention.  ``measure`` composes batches as the simulated scheduler does, under an
instance's limits, plans each and runs each layer's append and attention on a paged key/value cache
(``PagedKV``), times them, and ``fit`` turns the times into the attention's share of the
coefficients -- d and e in full, and its part of a, b and c, to which the caller adds what
the model's other layers take.  They go to ``LarContext.load_state`` as they are (ms).

    python -m paper_2607_18253_amd.calibrate --layers 32 --cache e4m3
"""

from __future__ import annotations

import argparse
from dataclasses import dataclass

import numpy as np

from .kv import PagedKV

NAMES = "abcde"
SHORTEST = 16  # prompt


@dataclass
class Instance:
    """Geometry and scheduler limits of a model instance (lar_kv_config, lar_sched_limits); a
    chunk_cap of 0 is none.  What runs on a GPU has a number of pages and a longest context."""
    n_q_heads: int = 32
    n_kv_heads: int = 8
    head_dim: int = 128
    layers: int = 32
    token_budget: int = 4096
    max_seqs: int = 256
    chunk_cap: int = 512
    kv_blocks: int = 18432
    block_size: int = 16
    max_ctx: int = 8192

    def __post_init__(self):
        if self.token_budget < 1 or self.max_seqs < 1 or self.chunk_cap < 0:
            raise ValueError("token_budget and max_seqs must be positive, chunk_cap not negative")
        if self.max_ctx < 2 or self.kv_blocks * self.block_size < min(self.max_ctx, SHORTEST):
            raise ValueError(f"max_ctx must be at least 2, and the pages hold a context of {SHORTEST} tokens or of max_ctx")

    @property
    def chunk(self):
        """The most tokens of a prompt in a batch."""
        return self.chunk_cap or self.token_budget


@dataclass
class Batch:
    """A token batch: new tokens and context (with them) per sequence, decodes first."""
    q_len: np.ndarray
    ctx_len: np.ndarray
    n_dec: int

    def features(self):
        """(1, P, D, C, A) of lar_instance_params' batch time: contexts are those before the batch."""
        q, before = self.q_len.astype(np.int64), self.ctx_len.astype(np.int64) - self.q_len
        n = self.n_dec
        chunk, at = q[n:], before[n:]
        return (1, int(chunk.sum()), n, int(before[:n].sum()),
                int((chunk * at + chunk * (chunk + 1) // 2).sum()))


def compose(inst: Instance, rng, n_dec: int, prompts) -> Batch:
    """A batch as the scheduler composes it: one token of each of n_dec decoding sequences,
    then chunks of the prompts in order, at most chunk_cap each where there is one, while the budget, the
    sequences and the pages last."""
    S = inst.block_size
    blocks, q, ctx = inst.kv_blocks, [], []
    for _ in range(min(n_dec, inst.max_seqs, inst.token_budget)):
        c = int(rng.integers(2, inst.max_ctx + 1))
        if -(-c // S) > blocks:
            break
        blocks -= -(-c // S)
        q.append(1)
        ctx.append(c)
    n, left = len(q), inst.token_budget - len(q)
    for p in prompts:
        done = int(rng.integers(0, p)) // inst.chunk * inst.chunk  # chunks of it before this one
        chunk = min(p - done, inst.chunk, left)
        if chunk < 1 or len(q) == inst.max_seqs or -(-(done + chunk) // S) > blocks:
            break
        blocks -= -(-(done + chunk) // S)
        left -= chunk
        q.append(chunk)
        ctx.append(done + chunk)
    return Batch(np.array(q, np.int32), np.array(ctx, np.int32), n)


def batches(inst: Instance, count: int, seed: int = 0):
    """Batches over the range an instance runs: from a few sequences to full ones, decodes
    alone, prefills alone and both."""
    rng = np.random.default_rng(seed)
    out = []
    while len(out) < count:
        kind = len(out) % 3
        n_dec = 0 if kind == 1 else int(rng.integers(1, min(inst.max_seqs, inst.token_budget) + 1))
        room = (inst.token_budget - n_dec) // inst.chunk + 1
        n_pre = 0 if kind == 0 else int(rng.integers(1, room + 1))
        prompts = np.clip(np.rint(rng.lognormal(6.5, 1.0, n_pre)), SHORTEST, inst.max_ctx - 1).astype(int)
        b = compose(inst, rng, n_dec, prompts)
        if len(b.q_len):
            out.append(b)
    return out


def fill(pages, generator):
    """Normal values into pages, as a running program's rows: what values toggle decides how fast a
    GPU under full load may run (a 7681-token chunk at 131072 takes 11.5 ms on zeros, 15 on these)."""
    import torch
    for t, exp in ((pages.k, pages.k_exp), (pages.v, pages.v_exp)):
        if exp is None:
            t.normal_(generator=generator)
            continue
        exp.fill_(127 - 7)   # of rows whose largest magnitude is 1.75 to 3.5
        step = max(1, (1 << 28) // t[0].numel())
        for a in range(0, len(t), step):
            part = t[a:a + step]
            part.copy_(torch.randn(part.shape, device=t.device, generator=generator).mul_(128).clamp_(-448, 448))


def measure(inst: Instance, sample, *, e4m3: bool = False, dtype=None, seed: int = 0, repeat: int = 3):
    """Milliseconds that the plan and all layers' append and attention of each batch take (the median of
    `repeat` runs), on pages dealt out in random order.  Needs memory for the pages of all
    layers."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    tokens = max(int(b.q_len.sum()) for b in sample)
    kv = PagedKV(inst.n_q_heads, inst.n_kv_heads, inst.head_dim, block_size=inst.block_size, dtype=dtype,
                 cache_dtype=torch.float8_e4m3fn if e4m3 else dtype, max_seqs=inst.max_seqs, max_tokens=tokens)
    dev, S = kv.device, inst.block_size
    g = torch.Generator(device=dev).manual_seed(seed)
    rng = np.random.default_rng(seed)
    # each layer's own, as in a model: a batch's contexts are not in a cache from the layer before
    layers = [kv.new_pages(inst.kv_blocks) for _ in range(inst.layers)]
    for pages in layers:   # contexts of earlier batches
        fill(pages, g)
    new = lambda heads: torch.randn((tokens, heads, inst.head_dim), device=dev, generator=g).to(dtype)
    q, k, v = new(inst.n_q_heads), new(inst.n_kv_heads), new(inst.n_kv_heads)
    out = torch.empty_like(q)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    times = []
    with kv:
        for b in sample:
            need = -(-b.ctx_len // S)
            table = np.zeros((len(need), int(need.max())), np.int32)
            free = rng.permutation(inst.kv_blocks)[:int(need.sum())]
            at = np.concatenate([[0], np.cumsum(need)])
            for s, n in enumerate(need):
                table[s, :n] = free[at[s]:at[s + 1]]
            tab = torch.from_numpy(table).to(dev)
            T = int(b.q_len.sum())
            got = []
            for _ in range(repeat + 1):   # the first one warms up
                start.record()
                kv.plan(b.q_len, b.ctx_len)
                for pages in layers:
                    kv.append(pages, k[:T], v[:T], tab)
                    kv.attend(pages, q[:T], tab, out=out[:T])
                end.record()
                end.synchronize()
                got.append(start.elapsed_time(end))
            times.append(sorted(got[1:])[repeat // 2])
        kv.sync()
    return np.array(times)


def fit(features, ms):
    """Coefficients a .. e >= 0 that take the features [n][5] to the times, least squares of
    the relative errors; terms that no batch has, and those that would come out negative,
    are 0."""
    X, y = np.asarray(features, np.float64), np.asarray(ms, np.float64)
    w = 1.0 / np.maximum(y, 1e-12)
    size = np.abs(X).max(0)
    use = list(np.nonzero(size)[0])
    while use:
        A = X[:, use] / size[use] * w[:, None]
        c = np.linalg.lstsq(A, y * w, rcond=None)[0]
        if (c >= 0).all():
            out = np.zeros(X.shape[1])
            out[use] = c / size[use]
            return out
        use.pop(int(np.argmin(c)))
    return np.zeros(X.shape[1])


def main(argv=None):
    import torch
    from .lar import LarContext
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("n_q_heads", 32), ("n_kv_heads", 8), ("head_dim", 128), ("layers", 32),
                          ("token_budget", 4096), ("max_seqs", 256), ("chunk_cap", 512), ("kv_blocks", 18432),
                          ("block_size", 16), ("max_ctx", 8192)):
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=default)
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--batches", type=int, default=48)
    a = vars(ap.parse_args(argv))
    e4m3, count = a.pop("cache") == "e4m3", a.pop("batches")
    inst = Instance(**a)
    sample = batches(inst, count)
    X = np.array([b.features() for b in sample])
    ms = measure(inst, sample, e4m3=e4m3)
    c = fit(X, ms)
    for n, v in zip(NAMES, c):
        print(f"{n} = {v:.6g} ms")
    print(f"mean relative error over {len(ms)} batches: {np.mean(np.abs(X @ c - ms) / ms):.3f}")
    # the simulation on them: one idle instance, prompts of several lengths
    with LarContext(1, 1, max_seqs_cap=inst.max_seqs, queue_cap=16, max_prompt=inst.max_ctx) as ctx:
        none = np.zeros(0, np.int32)
        ctx.load_state(a=c[:1], b=c[1:2], c=c[2:3], d=c[3:4], e=c[4:5], budget=[inst.token_budget],
                       max_seqs=[min(inst.max_seqs, inst.token_budget)], col=[0], offsets=[0, 0], rem_prefill=none, rem_decode=none,
                       context=none, clock_ms=[0.0])
        prompts = [p for p in (128, 1024, 8191) if p < inst.max_ctx]
        ttft, _ = ctx.estimate(torch.tensor(prompts, dtype=torch.int32, device="cuda"), 0.0)
        ctx.sync()
        for p, t in zip(prompts, ttft.flatten().tolist()):
            print(f"attention's part of an idle instance's TTFT, {p}-token prompt: {t:.3f} ms")
    return c


if __name__ == "__main__":
    main()
