"""What the calibration measures: the batches as a serving program runs them."""

from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2607_18253_amd import PagedKV  # noqa: E402
from paper_2607_18253_amd import calibrate as K  # noqa: E402

REPEAT, LAYERS = 2, 3


@pytest.fixture(params=[False, True], ids=["bf16", "e4m3"])
def run(request, monkeypatch):
    """(calls in order, pages) of a measurement of three batches."""
    calls, seen = [], {}

    class Noted(PagedKV):
        def plan(self, *a, **k):
            calls.append("plan")
            return super().plan(*a, **k)

        def append(self, pages, *a, **k):
            calls.append(("append", pages.k.data_ptr()))
            seen[pages.k.data_ptr()] = pages
            return super().append(pages, *a, **k)

        def attend(self, pages, *a, **k):
            calls.append(("attend", pages.k.data_ptr()))
            return super().attend(pages, *a, **k)

    class Event(torch.cuda.Event):
        def record(self, *a):
            calls.append("record")
            return super().record(*a)
    monkeypatch.setattr(K, "PagedKV", Noted)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    inst = K.Instance(n_q_heads=8, n_kv_heads=2, head_dim=64, layers=LAYERS, token_budget=256, max_seqs=24, chunk_cap=64,
                      kv_blocks=600, max_ctx=512)
    ms = K.measure(inst, K.batches(inst, 3, seed=2), e4m3=request.param, repeat=REPEAT)
    assert (ms > 0).all()
    return calls, list(seen.values())


def values(t, exp):
    x = t.float()
    return x if exp is None else x * torch.exp2(exp.float() - 127)[..., None]


def test_contexts_hold_values(run):
    """Finite values of unit size, of which no two tokens' rows are alike, K and V not alike."""
    for p in run[1]:
        k, v = values(p.k, p.k_exp), values(p.v, p.v_exp)
        assert torch.isfinite(k).all() and torch.isfinite(v).all()
        assert 0.5 < k.std() < 2.0 and 0.5 < v.std() < 2.0 and abs(k.mean()) < 0.1
        assert not torch.equal(k, v) and len(torch.unique(k.flatten(0, 2), dim=0)) > 0.9 * k.flatten(0, 2).shape[0]


def test_layers_have_their_own_pages(run):
    at = [c[1] for c in run[0] if c[0] == "attend"]
    assert len(set(at)) == LAYERS == len(run[1])
    assert all(len(set(at[i:i + LAYERS])) == LAYERS for i in range(0, len(at), LAYERS))
    ends = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for p in run[1] for t in p.tensors())
    assert all(a[1] <= b[0] for a, b in zip(ends, ends[1:]))


def test_a_batch_is_timed_with_its_plan(run):
    calls = [c if isinstance(c, str) else c[0] for c in run[0]]
    one = ["record", "plan"] + ["append", "attend"] * LAYERS + ["record"]
    timed = "|".join(calls)
    assert timed.count("|".join(one)) == 3 * (REPEAT + 1)


def test_more_sequences_than_budget(capsys):
    """The command on an instance whose batches cannot hold a token of every sequence."""
    c = K.main(["--layers", "2", "--token-budget", "128", "--max-seqs", "256", "--kv-blocks", "2000", "--max-ctx", "2048",
                "--batches", "9"])
    assert (c >= 0).all() and "1024-token prompt" in capsys.readouterr().out
