"""Refusals of the 8-bit cache and of adjusted logits, on the CPU: every invalid argument returns its
documented code before anything is launched, with the plain library and with its host code under
AddressSanitizer and UndefinedBehaviorSanitizer."""

import ctypes
import os

import pytest

from paper_2606_03681_amd import tfm

FAKE, FAR, BIG = 1 << 20, 1 << 60, 1 << 50
NAN, INF = float("nan"), float("inf")


def _cache(**kw):
    base = dict(heads=2, d=32, page=64, n_pages=10)
    base.update(kw)
    return tfm.make_cache8(**base)


def _rows(**kw):
    base = dict(B=3, L=5, max_pages=4, dtype="bf16", stride_k=(5 * 64, 64, 32),
                stride_v=(5 * 64, 64, 32))
    base.update(kw)
    return tfm.make_cache8_rows(**base)


def _query(**kw):
    base = dict(B=3, L=5, heads=4, max_pages=4, dtype="bf16", stride_q=(5 * 128, 128, 32),
                stride_out=(5 * 128, 128, 32), scale=0.2, causal=True, max_len=0)
    base.update(kw)
    return tfm.make_cache8_query(**base)


def _append(c=None, r=None, k=FAKE, v=FAKE, pages=FAKE, lens=FAKE, n_new=FAKE, pool=FAR, nb=BIG):
    c, r = c or _cache(), r or _rows()
    return tfm.lib().tfm_cache8_append(ctypes.byref(c), ctypes.byref(r), k, v, pages, lens, n_new,
                                       pool, nb, None)


def _attend(c=None, a=None, q=FAKE, pages=FAKE, lens=FAKE, n_rows=FAKE, pool=FAR, nb=BIG,
            out=FAKE << 8, lse=FAKE << 16, ws=FAKE, wb=BIG):
    c, a = c or _cache(), a or _query()
    return tfm.lib().tfm_cache8_attend(ctypes.byref(c), ctypes.byref(a), q, pages, lens, n_rows,
                                       pool, nb, out, lse, ws, wb, None)


@pytest.mark.parametrize("kw,code", [
    (dict(heads=0), -1), (dict(heads=4097), -1), (dict(d=0), -2), (dict(d=24), -2),
    (dict(d=256), -2), (dict(page=0), -1), (dict(page=8), -1), (dict(page=48), -1),
    (dict(page=512), -1), (dict(n_pages=0), -1), (dict(n_pages=-1), -1),
    (dict(heads=4096, d=128, page=256, n_pages=1 << 20), -1),
])
def test_pools_refused(kw, code):
    c = _cache(**kw)
    assert tfm.cache8_bytes(c) == 0
    assert _append(c) == code and _attend(c, _query(heads=4096)) == code
    assert tfm.cache8_attend_workspace_bytes(c, _query()) == 0
    assert tfm.last_error()


def test_pool_bytes():
    for c in (_cache(), _cache(heads=1, d=16, page=16, n_pages=1), _cache(page=256, d=128)):
        assert tfm.cache8_bytes(c) == c.n_pages * c.heads * (2 * c.page * c.d + 2)
    assert tfm.cache8_bytes(_cache(n_pages=2 ** 31 - 1, heads=1, d=16, page=16)) > 2 ** 39


@pytest.mark.parametrize("kw", [
    dict(B=-1), dict(L=-1), dict(max_pages=-1), dict(max_pages=(1 << 30) // 64 + 1),
    dict(B=1 << 16, max_pages=1 << 15), dict(dtype=2), dict(stride_k=(-1, 64, 32)),
    dict(stride_v=(0, (1 << 40) + 1, 0)), dict(B=1 << 20, stride_k=(1 << 40, 0, 0)),
])
def test_rows_refused(kw):
    assert _append(r=_rows(**kw)) == -1
    assert tfm.last_error()


@pytest.mark.parametrize("kw", [
    dict(B=-1), dict(L=-1), dict(max_pages=-1), dict(max_pages=(1 << 30) // 64 + 1), dict(dtype=-1),
    dict(heads=0), dict(heads=3), dict(heads=(1 << 16) + 2), dict(B=1 << 16, L=1 << 15),
    dict(B=1, L=1 << 25), dict(max_len=-1), dict(scale=NAN), dict(scale=INF), dict(scale=-INF),
    dict(scale=2.0 ** 64 * 1.001), dict(scale=-3e38), dict(stride_q=(0, -1, 0)),
    dict(stride_out=(5 * 128, 128, 31)), dict(stride_out=(5 * 128, 100, 32)),
    dict(stride_out=(100, 128, 32)), dict(stride_out=(0, 128, 32)),
    dict(stride_q=((1 << 40) + 1, 0, 0)),
])
def test_queries_refused(kw):
    a = _query(**kw)
    assert tfm.cache8_attend_workspace_bytes(_cache(), a) == 0
    assert _attend(a=a) == -1
    assert tfm.last_error()


def test_cache_pointers_and_buffers_refused():
    for bad in (dict(k=0), dict(v=0), dict(k=FAKE + 1), dict(v=FAKE + 1), dict(pages=FAKE + 2),
                dict(lens=FAKE + 2), dict(n_new=FAKE + 1), dict(pool=0), dict(pool=FAR + 8)):
        assert _append(**bad) == -5, bad
    need = tfm.cache8_bytes(_cache())
    assert _append(nb=need - 1) == -7 and _attend(nb=need - 1) == -7
    for bad in (dict(q=0), dict(out=0), dict(lens=0), dict(q=FAKE + 1), dict(out=FAKE + 1),
                dict(lens=FAKE + 2), dict(pages=FAKE + 2), dict(n_rows=FAKE + 1),
                dict(lse=FAKE + 2), dict(pool=0), dict(pool=FAR + 8)):
        assert _attend(**bad) == -5, bad
    # what is written shares nothing with what is read
    assert _append(k=FAR + 64) == -5 and "overlaps" in tfm.last_error()
    assert _append(v=FAR - 64) == -5
    assert _attend(out=FAR + 64) == -5 and "overlaps" in tfm.last_error()
    assert _attend(lse=(FAKE << 8) + 4) == -5 and _attend(lse=FAR + 16) == -5
    assert _attend(a=_query(stride_q=(0, 128, 32)), out=FAKE) == -5
    lib = tfm.lib()
    c, r, a = (ctypes.byref(x) for x in (_cache(), _rows(), _query()))
    assert lib.tfm_cache8_bytes(None) == 0
    assert lib.tfm_cache8_append(None, r, *[FAKE] * 6, BIG, None) == -5
    assert lib.tfm_cache8_append(c, None, *[FAKE] * 6, BIG, None) == -5
    assert lib.tfm_cache8_attend(None, a, *[FAKE] * 5, BIG, FAKE, FAKE, FAKE, BIG, None) == -5
    assert lib.tfm_cache8_attend(c, None, *[FAKE] * 5, BIG, FAKE, FAKE, FAKE, BIG, None) == -5
    assert lib.tfm_cache8_attend_workspace_bytes(c, None) == 0


def test_a_workspace_that_is_too_small_is_refused():
    c = _cache(heads=1, d=128, n_pages=3000)
    a = _query(B=1, L=1, heads=1, max_pages=3000, stride_q=(0, 0, 0), stride_out=(0, 0, 0))
    need = tfm.cache8_attend_workspace_bytes(c, a)
    if need:
        assert _attend(c, a, ws=0) == -5 and _attend(c, a, ws=FAKE + 8) == -5
        assert _attend(c, a, wb=need - 1) == -7


def test_nothing_to_do_needs_no_rows():
    for kw in (dict(B=0), dict(L=0)):
        assert _append(r=_rows(**kw), k=0, v=0, lens=0, pages=0, n_new=0) == 0
        assert _attend(a=_query(**kw), q=0, out=0, lens=0, lse=0, ws=0, wb=0) == 0
    assert _append(r=_rows(max_pages=0)) == 0


_A = ("logits", "n_class", "history", "n_history", "repetition", "presence", "frequency",
      "bias_idx", "bias", "allowed", "out")


def _adjust(**kw):
    base = dict(N=4, V=100, ld=100, dtype="bf16", n_hist=7, n_bias=3)
    base.update(kw)
    return tfm.make_adjust(**base)


def _call(a, **kw):
    ptrs = {n: (i + 1) * (FAKE << 8) for i, n in enumerate(_A)}
    ptrs.update(kw)
    return tfm.lib().tfm_adjust_logits(ctypes.byref(a), *[ptrs[n] for n in _A], None)


@pytest.mark.parametrize("kw", [
    dict(N=-1), dict(N=(1 << 27) + 1), dict(V=0), dict(V=(1 << 18) + 1, ld=1 << 19), dict(ld=99),
    dict(ld=(1 << 40) + 1), dict(ld_out=99), dict(dtype=2), dict(n_hist=-1), dict(n_bias=-1),
    dict(n_hist=(1 << 27) + 1), dict(n_bias=(1 << 27) + 1), dict(ld_history=6), dict(ld_bias=2),
    dict(ld_allowed=3), dict(ld_allowed=-1), dict(ld_history=(1 << 40) + 1),
    dict(N=1 << 20, ld_bias=1 << 40), dict(N=1 << 20, ld=1 << 40),
])
def test_adjustment_dims_refused(kw):
    assert _call(_adjust(**kw)) == -1
    assert tfm.last_error()


def test_adjustment_pointers_refused():
    a = _adjust()
    for name in ("logits", "out", "history", "bias_idx", "bias"):
        assert _call(a, **{name: 0}) == -5, name
    for name in _A:
        assert _call(a, **{name: (FAKE << 6) + 1}) == -5, name
    at = FAKE << 8
    assert _call(a, logits=at, out=at + 16) == -5 and "overlaps" in tfm.last_error()
    assert _call(_adjust(ld_out=101), logits=at, out=at) == -5
    for name in _A[1:-1]:
        assert _call(a, **{name: (FAKE << 8) * 11}) == -5, name     # where out is
        assert name in tfm.last_error()
    assert tfm.lib().tfm_adjust_logits(None, *[FAKE] * 11, None) == -5
    assert _call(_adjust(N=0), **{n: 0 for n in _A}) == 0


def _dims(**kw):
    base = dict(B=2, R=64, C=8, E=64, heads=4, H=128, dtype="bf16")
    base.update(kw)
    return tfm.make_dims(**base)


def test_layer_calls_with_8_bit_caches_refused():
    import numpy as np
    lib, mask = tfm.lib(), np.ones((2, 9), np.uint8)

    def ctx(d=None, nt=(5, 5), ptr=FAKE, pool=FAKE, cb=BIG, pb=BIG, wb=BIG):
        n = np.array(nt, np.int32)
        return lib.tfm_layer_fwd_context8(ctypes.byref(d or _dims()), n.ctypes.data,
                                          mask.ctypes.data, FAKE, FAKE, FAKE, ptr, cb, pool, pb,
                                          FAKE, wb, None)

    def qry(rc, d=None, nt=(5, 5), pool=FAKE, pb=BIG, wb=BIG):
        n = np.array(nt, np.int32)
        return lib.tfm_layer_fwd_query8(ctypes.byref(d or _dims(R=8)), rc, n.ctypes.data,
                                        mask.ctypes.data, FAKE, FAKE, pool, pb, FAKE, FAKE, wb, None)

    assert ctx(_dims(dtype="f32")) == -1 and ctx(nt=(5, 65)) == -3
    assert ctx(ptr=0) == -5 and ctx(pool=0) == -5 and ctx(pool=FAKE + 8) == -5
    need = tfm.infer_cache8_bytes(_dims())
    assert need == 2 * 9 * 4 * (2 * 64 * 16 + 2)
    assert ctx(cb=16) == -7 and ctx(wb=16) == -7 and ctx(pb=need - 1) == -7
    assert "cache8" in tfm.last_error()
    assert qry(0) == -1 and qry(-3) == -1 and qry(32, nt=(5, 33)) == -3
    assert qry(32, pool=0) == -5 and qry(32, pool=FAKE + 2) == -5
    assert qry(100, pb=tfm.infer_cache8_bytes(_dims(R=100)) - 1) == -7
    assert qry(32, wb=tfm.infer8_workspace_bytes(_dims(R=8), 32) - 1) == -7
    assert tfm.infer_cache8_bytes(_dims(dtype="f32")) == 0
    assert tfm.infer8_workspace_bytes(_dims(dtype="f32"), 32) == 0
    assert tfm.infer8_workspace_bytes(_dims(), 0) == 0
    for rows in (1, 8, 64, 300):
        for rc in (1, 64, 700, 5000):
            assert tfm.infer8_workspace_bytes(_dims(R=rows), rc) >= \
                tfm.infer_workspace_bytes(_dims(R=rows))


def test_binding_refuses_tensors_that_do_not_fit():
    """The Python calls look at types and shapes first (no GPU is touched for these)."""
    import torch
    i32 = torch.int32
    c = _cache()
    pool = torch.zeros(tfm.cache8_bytes(c), dtype=torch.uint8)
    k = torch.zeros((3, 5, 2, 32), dtype=torch.bfloat16)
    pages, lens = torch.zeros((3, 4), dtype=i32), torch.zeros(3, dtype=i32)
    for bad in ((k.float(), k, pages, lens, None), (k, k[:2].clone(), pages, lens, None),
                (k, k, pages[:2], lens, None), (k, k, pages.long(), lens, None),
                (k, k, pages, lens[:2], None), (k, k, pages, lens, lens.long()),
                (k, k, pages, lens, lens)):
        with pytest.raises(ValueError):          # the last one: not on the GPU
            tfm.cache8_append(c, _rows(), *bad, pool)
    q, lse = torch.zeros((3, 5, 4, 32), dtype=torch.bfloat16), torch.zeros((3, 5, 4))
    for bad in ((q.float(), pages, lens, q, lse), (q, pages, lens, q[:2].clone(), lse),
                (q, pages, lens, q, lse[:2]), (q, pages, lens, q, lse.double()),
                (q, pages.t(), lens, q, lse), (q, pages, lens, q, lse)):
        with pytest.raises(ValueError):
            tfm.cache8_attend(c, _query(), bad[0], bad[1], bad[2], None, pool, bad[3], bad[4], None)
    with pytest.raises(ValueError):
        tfm.make_cache8_rows(1, 1, 1, "f32", (0, 0), (0, 0, 0))
    with pytest.raises(ValueError):
        tfm.make_cache8_query(1, 1, 1, 1, "f32", (0, 0, 0), (0, 0), 1.0)
    z, h = torch.zeros((4, 100), dtype=torch.bfloat16), torch.zeros((4, 7), dtype=i32)
    b, m = torch.zeros((4, 3)), torch.zeros((4, 4), dtype=i32)
    good = dict(logits=z, n_class=None, history=h, n_history=None, repetition=None, presence=None,
                frequency=None, bias_idx=b.int(), bias=b, allowed=m, out=z)
    for bad in (dict(logits=z.float()), dict(out=z[:, :99]), dict(history=h[:3].clone()),
                dict(bias=b.double()), dict(allowed=m[:, :3].clone()), dict(history=h.long()),
                dict(presence=torch.zeros(3)), dict(allowed=torch.zeros((4, 8), dtype=i32)[:, ::2]),
                dict()):
        with pytest.raises(ValueError):
            tfm.adjust_logits(_adjust(), **{**good, **bad})


def test_refusals_clean_under_sanitizers():
    if os.environ.get("TFM_LIB"):
        pytest.skip("already in the sanitized child")
    from test_host_sanitized import _run
    from paper_2606_03681_amd import build
    env = dict(os.environ, LD_PRELOAD=build.san_runtime(), TFM_LIB=build.build(sanitize=True),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    rc, out = _run(env, ["-m", "pytest", "-q", "-p", "no:cacheprovider",
                         os.path.join("tests", "test_cache_abi_cpu.py")])
    assert rc == 0, out[-6000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-6000:]
