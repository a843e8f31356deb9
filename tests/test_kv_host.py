"""CPU-side checks of the paged key/value cache's entry points and of the calibration (no
GPU calls)."""

import ctypes as C
import os

import numpy as np
import pytest

from test_kernel_resources import LIB, kernels  # noqa: F401  (the fixture)


def test_null_arguments_rejected_without_gpu():
    if not os.path.exists(LIB):
        pytest.skip("liblar.so not built")
    lib = C.CDLL(LIB)
    out = C.c_void_p(1)
    assert lib.lar_kv_create(None, None) == -1
    assert lib.lar_kv_create(C.byref(out), None) == -1 and out.value is None
    assert lib.lar_kv_destroy(None) == 0
    assert lib.lar_kv_sync(None) == -1
    assert lib.lar_kv_plan(None, 1, None, None, 0, 0) == -1
    for name, n in (("lar_kv_append", 6), ("lar_kv_read", 6)):
        assert getattr(lib, name)(*[None] * n) == -1, name
    lib.lar_kv_attend.argtypes = [C.c_void_p] * 4 + [C.c_int32, C.c_double, C.c_void_p, C.c_void_p]
    assert lib.lar_kv_attend(None, None, None, None, 1, 1.0, None, None) == -1
    lib.lar_kv_error_string.restype = C.c_char_p
    assert lib.lar_kv_error_string(None) == b"null handle"


@pytest.mark.parametrize("field,value", [
    ("n_q_heads", 7), ("n_q_heads", 0), ("n_q_heads", 130), ("n_kv_heads", 0), ("n_kv_heads", -2), ("head_dim", 96),
    ("dtype", 2), ("dtype", 5), ("cache_dtype", 0), ("block_size", 0), ("block_size", 48), ("block_size", 1 << 17),
    ("max_seqs", 0), ("max_tokens", 0), ("max_tokens", 1 << 27), ("max_tokens", (1 << 26) + 1), ("reserved", 1)])
def test_bad_configurations_rejected_without_gpu(field, value):
    if not os.path.exists(LIB):
        pytest.skip("liblar.so not built")
    from paper_2607_18253_amd.kv import KvConfig
    lib = C.CDLL(LIB)
    cfg = KvConfig(8, 2, 128, 1, 1, 16, 4, 64, 0, None)
    setattr(cfg, field, value)
    out = C.c_void_p(1)
    assert lib.lar_kv_create(C.byref(out), C.byref(cfg)) == -1
    assert out.value is None


def test_cache_kernels_keep_their_registers(kernels):  # noqa: F811
    """The cache's kernels use no scratch memory, and the wide ones' workgroups fit a CU."""
    names = [n for n in kernels if "k_kv_" in n]
    assert sum("k_kv_wide" in n for n in names) == 16 and sum("k_kv_narrow" in n for n in names) == 8
    for n in names:
        k = kernels[n]
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n
        assert k[".group_segment_fixed_size"] <= 160 * 1024, n
        if "k_kv_wide" in n or "k_kv_narrow" in n:
            assert k[".vgpr_count"] <= 256, n


# ------------------------------------------------------------------ calibration
def test_batches_hold_the_limits():
    from paper_2607_18253_amd import calibrate as K
    inst = K.Instance(token_budget=300, max_seqs=40, chunk_cap=64, kv_blocks=700, block_size=16, max_ctx=512)
    some = K.batches(inst, 60, seed=3)
    for b in some:
        assert b.q_len.sum() <= inst.token_budget and len(b.q_len) <= inst.max_seqs
        assert (b.q_len[:b.n_dec] == 1).all() and (b.q_len <= inst.chunk_cap).all() and (b.q_len >= 1).all()
        assert (b.ctx_len >= b.q_len).all() and (b.ctx_len <= inst.max_ctx).all()
        assert (-(-b.ctx_len // inst.block_size)).sum() <= inst.kv_blocks
    assert any(b.n_dec == 0 for b in some) and any(b.n_dec == len(b.q_len) for b in some)
    assert any(0 < b.n_dec < len(b.q_len) for b in some)


def test_features_count_token_by_token():
    """P, D, C, A of the batch time, against counting each new token's own context."""
    from paper_2607_18253_amd import calibrate as K
    b = K.Batch(np.array([1, 1, 3, 5], np.int32), np.array([10, 2, 3, 25], np.int32), 2)
    A = sum(j + 1 for j in range(3)) + sum(20 + j + 1 for j in range(5))
    assert b.features() == (1, 8, 2, 9 + 1, A)


def test_fit_recovers_the_coefficients():
    from paper_2607_18253_amd import calibrate as K
    inst = K.Instance()
    X = np.array([b.features() for b in K.batches(inst, 40, seed=1)])
    want = np.array([0.3, 1e-4, 2e-3, 4e-6, 3e-7])
    np.testing.assert_allclose(K.fit(X, X @ want), want, rtol=1e-6)
    # a term that only noise would make negative is left out, and absent ones are 0
    y = X @ np.array([0.5, 0.0, 0.0, 1e-6, 0.0])
    c = K.fit(X, y * (1 + 1e-3 * np.sin(np.arange(len(y)))))
    assert (c >= 0).all() and abs(c[3] / 1e-6 - 1) < 0.02
    X[:, 4] = 0
    assert K.fit(X, X @ want)[4] == 0


def test_lengths_are_not_cut():
    """Lengths that 32 bits cannot hold, fractions and tables are refused, not rounded."""
    from paper_2607_18253_amd.kv import _int32s
    for ok in ([], [1, 2], np.array([3], np.int64), np.array([7, 2 ** 31 - 1], np.uint32), (4,)):
        assert _int32s(ok, "x").dtype == np.int32 and _int32s(ok, "x").tolist() == [int(v) for v in ok]
    for bad in ([2 ** 31], [2 ** 32 + 5], [-2 ** 31 - 1], [1.5], [2.0], [[1, 2]], 3, np.array([2 ** 40]), [2 ** 70]):
        with pytest.raises(ValueError):
            _int32s(bad, "x")
