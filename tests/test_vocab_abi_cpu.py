"""Refusals of the operators over discrete values, on the CPU: every invalid argument returns its
documented code before anything is launched, with the plain library and with its host code under
AddressSanitizer and UndefinedBehaviorSanitizer."""

import ctypes
import os

import numpy as np
import pytest

from paper_2606_03681_amd import tfm

FAKE, BIG = 1 << 20, 1 << 50


def _embed(**kw):
    base = dict(n=(2, 3, 4), stride=(1000, 200, 40), E=32, V=10, dtype="bf16", table_dtype="f32",
                scale=1.0)
    base.update(kw)
    return tfm.make_embed(**base)


def _fwd(e, ids=FAKE, table=FAKE, out=FAKE):
    return tfm.lib().tfm_embed_fwd(ctypes.byref(e), ids, table, out, 0, None)


def _bwd(e, ids=FAKE, dout=FAKE, dtable=FAKE, ws=FAKE, wb=BIG):
    return tfm.lib().tfm_embed_bwd(ctypes.byref(e), ids, dout, dtable, 0, ws, wb, None)


@pytest.mark.parametrize("kw", [
    dict(n=(-1, 3, 4)), dict(n=(1 << 10, 1 << 10, 1 << 8)), dict(n=(2 ** 31 - 1,) * 3),
    dict(V=0), dict(V=(1 << 24) + 1), dict(E=0), dict(E=(1 << 16) + 1), dict(dtype=2),
    dict(table_dtype=-1), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(stride=(-1, 200, 40)), dict(stride=((1 << 40) + 1, 200, 40)),
    dict(n=(1 << 20, 1, 1), stride=(1 << 40, 0, 0)),
])
def test_embedding_dims_refused(kw):
    e = _embed(**kw)
    assert tfm.embed_workspace_bytes(e) == 0
    assert _fwd(e) == -1 and _bwd(e) == -1
    assert tfm.last_error()


@pytest.mark.parametrize("stride", [(1000, 200, 31), (1000, 100, 40), (500, 200, 40), (0, 200, 40),
                                    (1000, 0, 40), (40, 41, 42)])
def test_embedding_rows_that_overlap_refused_in_the_forward(stride):
    assert _fwd(_embed(stride=stride)) == -1
    assert "overlap" in tfm.last_error()
    assert tfm.embed_workspace_bytes(_embed(stride=stride)) > 0    # the backward only reads


def test_embedding_pointers_and_workspace_refused():
    e = _embed()
    for bad in (dict(ids=0), dict(ids=FAKE + 2), dict(table=0), dict(table=FAKE + 2),
                dict(out=0), dict(out=FAKE + 1)):
        assert _fwd(e, **bad) == -5, bad
    for bad in (dict(ids=0), dict(dout=0), dict(dout=FAKE + 1), dict(dtable=0),
                dict(dtable=FAKE + 2), dict(ws=0), dict(ws=FAKE + 8)):
        assert _bwd(e, **bad) == -5, bad
    assert _bwd(e, wb=tfm.embed_workspace_bytes(e) - 1) == -7
    assert tfm.lib().tfm_embed_fwd(None, FAKE, FAKE, FAKE, 0, None) == -5
    assert tfm.lib().tfm_embed_bwd(None, FAKE, FAKE, FAKE, 0, FAKE, BIG, None) == -5


def test_embedding_of_nothing_needs_no_rows():
    assert _fwd(_embed(n=(2, 0, 4)), ids=0, table=0, out=0) == 0


def test_embedding_workspace_does_not_shrink_with_more_ids():
    sizes = [tfm.embed_workspace_bytes(_embed(n=(1, 1, n), stride=(0, 0, 32), V=V))
             for V in (10, 50021) for n in (0, 1, 100, 4096, 5000, 100000, 1 << 20)]
    assert all(s > 0 for s in sizes)
    assert sizes[:7] == sorted(sizes[:7]) and sizes[7:] == sorted(sizes[7:])


def _distill(**kw):
    base = dict(N=4, V=100, k=5, ld=100, dtype="bf16", temperature=2.0, alpha=1.0, tail=0)
    base.update(kw)
    return tfm.make_distill(**base)


_D = ("logits", "top_idx", "top_logit", "top_lse", "labels", "weights", "n_class", "loss",
      "row_loss", "dlogits")


def _loss(d, ws=FAKE, wb=BIG, **kw):
    ptrs = {n: (i + 1) * (FAKE << 8) for i, n in enumerate(_D)}
    ptrs.update(kw)
    return tfm.lib().tfm_distill_loss(ctypes.byref(d), *[ptrs[n] for n in _D], ws, wb, None)


@pytest.mark.parametrize("kw", [
    dict(N=-1), dict(N=(1 << 27) + 1), dict(V=0), dict(V=(1 << 18) + 1, ld=1 << 19), dict(ld=99),
    dict(ld=(1 << 40) + 1), dict(N=1 << 20, ld=1 << 40), dict(k=0), dict(k=257), dict(dtype=2),
    dict(tail=2), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
    dict(temperature=float("inf")), dict(alpha=-0.1), dict(alpha=1.5), dict(alpha=float("nan")),
])
def test_distillation_dims_refused(kw):
    d = _distill(**kw)
    assert tfm.distill_workspace_bytes(d) == 0
    assert _loss(d) == -1
    assert tfm.last_error()


def test_distillation_pointers_and_workspace_refused():
    d = _distill()
    for name in ("logits", "top_idx", "top_logit", "loss"):
        assert _loss(d, **{name: 0}) == -5, name
        assert _loss(d, **{name: FAKE + 1}) == -5, name
    for name in ("weights", "n_class", "row_loss", "dlogits"):
        assert _loss(d, **{name: FAKE + 1}) == -5, name
    assert _loss(_distill(tail=1), top_lse=0) == -5
    assert _loss(_distill(alpha=0.5), labels=0) == -5
    assert "labels" in tfm.last_error()
    # the gradient may be written over the logits, but not over part of them
    at = FAKE << 8
    assert _loss(d, logits=at, dlogits=at + 16) == -5
    assert _loss(d, logits=at, dlogits=at - 16) == -5
    assert "overlaps" in tfm.last_error()
    assert _loss(d, ws=0) == -5 and _loss(d, ws=FAKE + 4) == -5
    assert _loss(d, wb=tfm.distill_workspace_bytes(d) - 1) == -7
    assert tfm.lib().tfm_distill_loss(None, *[FAKE] * 10, FAKE, BIG, None) == -5


_S = ("logits", "n_class", "temperature", "top_k", "top_p", "min_p", "u", "token", "logprob")


def _sample(s, **kw):
    ptrs = {n: FAKE for n in _S}
    ptrs.update(kw)
    return tfm.lib().tfm_sample(ctypes.byref(s), *[ptrs[n] for n in _S], None)


def test_sampling_arguments_refused():
    good = dict(N=4, V=100, ld=100, dtype="f32")
    for kw in (dict(N=-1), dict(N=(1 << 27) + 1), dict(V=0), dict(V=(1 << 18) + 1, ld=1 << 19),
               dict(ld=99), dict(ld=(1 << 40) + 1), dict(N=1 << 20, ld=1 << 40), dict(dtype=3)):
        assert _sample(tfm.make_sampling(**{**good, **kw})) == -1, kw
        assert tfm.last_error()
    s = tfm.make_sampling(**good)
    for name in ("logits", "u", "token"):
        assert _sample(s, **{name: 0}) == -5, name
    for name in _S:
        assert _sample(s, **{name: FAKE + 2}) == -5, name
    assert tfm.lib().tfm_sample(None, *[FAKE] * 9, None) == -5
    assert _sample(tfm.make_sampling(**{**good, "N": 0}), **{n: 0 for n in _S}) == 0


def test_decoder_backward_arguments_refused():
    d = tfm.make_dims(B=2, R=64, C=8, E=64, heads=4, H=128, dtype="f32")
    en = tfm.make_ends(1, [0], 8, 0, 128, 10, 0)
    nt, nf = np.array([5, 6], np.int32), np.array([8, 8], np.int32)

    def call(nt=nt, nf=nf, ws=FAKE, wb=BIG, **kw):
        p = dict(Y=FAKE, params=FAKE, dlogits=FAKE, dY=FAKE, grads=FAKE)
        p.update(kw)
        return tfm.lib().tfm_decode_bwd(
            ctypes.byref(d), ctypes.byref(en), None if nt is None else nt.ctypes.data,
            None if nf is None else nf.ctypes.data, p["Y"], p["params"], p["dlogits"], p["dY"],
            p["grads"], 0, ws, wb, None)

    for name in ("Y", "params", "dlogits", "dY", "grads"):
        assert call(**{name: 0}) == -5 and call(**{name: FAKE + 4}) == -5, name
    assert call(nt=None) == -5 and call(nf=None) == -5
    assert call(nt=np.array([5, 65], np.int32)) == -3
    assert call(nt=np.array([-1, 5], np.int32)) == -3
    assert call(nf=np.array([0, 8], np.int32)) == -1
    assert call(ws=0) == -5 and call(wb=16) == -7


def test_binding_refuses_tensors_that_do_not_fit():
    """The Python calls look at types and shapes first (no GPU is touched for these)."""
    import torch
    e = _embed(n=(1, 1, 4), stride=(0, 0, 32))
    ids, table = torch.zeros((1, 1, 4), dtype=torch.int32), torch.zeros((10, 32))
    out = torch.zeros((4, 32), dtype=torch.bfloat16)
    for bad in ((ids.long(), table, out), (ids[..., :3], table, out),
                (ids, table.bfloat16(), out), (ids, table[:9], out), (ids, table.t(), out),
                (ids, table, out.float()), (ids, table, out[:3].clone()), (ids, table, out)):
        with pytest.raises(ValueError):          # the last one: not on the GPU
            tfm.embed_fwd(e, *bad)
    s = tfm.make_sampling(2, 8, 8, "f32")
    z, u, tok = torch.zeros((2, 8)), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for bad in ((z.double(), u, tok), (z[:, :7], u, tok), (z, u.double(), tok), (z, u[:1], tok),
                (z, u, tok.long()), (torch.zeros((2, 16))[:, ::2], u, tok)):
        with pytest.raises(ValueError):
            tfm.sample(s, bad[0], None, None, None, None, None, bad[1], bad[2])


def test_refusals_clean_under_sanitizers():
    if os.environ.get("TFM_LIB"):
        pytest.skip("already in the sanitized child")
    from test_host_sanitized import _run
    from paper_2606_03681_amd import build
    env = dict(os.environ, LD_PRELOAD=build.san_runtime(), TFM_LIB=build.build(sanitize=True),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    rc, out = _run(env, ["-m", "pytest", "-q", "-p", "no:cacheprovider",
                         os.path.join("tests", "test_vocab_abi_cpu.py")])
    assert rc == 0, out[-6000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-6000:]


@pytest.mark.parametrize("tau", [1e-45, 4e-39, 2.0 ** -21, 1.01 * 2.0 ** 20, 1e30, 3e38])
def test_distillation_temperatures_refused(tau):
    """Temperatures at which 1 / tau or tau^2 D leaves float32's range or precision."""
    assert tfm.distill_workspace_bytes(_distill(temperature=tau)) == 0
    assert _loss(_distill(temperature=tau)) == -1
    assert "temperature" in tfm.last_error()
    for ok in (2.0 ** -20, 2.0 ** 20):
        assert tfm.distill_workspace_bytes(_distill(temperature=ok)) > 0


def test_binding_leaves_a_missing_workspace_to_the_library():
    """No workspace: the library's own refusal (on the GPU for the calls that look at devices first,
    as here), not an error on the way to it."""
    import torch
    e, ids = _embed(n=(1, 1, 4), stride=(0, 0, 32)), torch.zeros((1, 1, 4), dtype=torch.int32)
    rows, table = torch.zeros((4, 32), dtype=torch.bfloat16), torch.zeros((10, 32))
    with pytest.raises(ValueError, match="not on the current GPU"):
        tfm.embed_bwd(e, ids, rows, table, False, None)
    d = _distill(N=2, V=8, k=1, ld=8)
    z, one = torch.zeros((2, 8), dtype=torch.bfloat16), torch.zeros((2, 1))
    with pytest.raises(ValueError, match="not on the current GPU"):
        tfm.distill_loss(d, z, one.int(), one, None, None, None, None, torch.zeros(1), None, z, None)
    dims = tfm.make_dims(B=2, R=64, C=8, E=64, heads=4, H=128, dtype="f32")
    with pytest.raises(tfm.TfmError, match="workspace"):
        tfm.decode_bwd(dims, tfm.make_ends(1, [0], 8, 0, 128, 10, 0), [5, 6], [8, 8], FAKE, FAKE,
                       FAKE, FAKE, FAKE, False, None, stream=0)


def test_current_stream_with_and_without_the_raw_handle(monkeypatch):
    """The binding takes the current stream's handle from whichever call torch has."""
    import types

    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 100 + d, raising=False)
    assert tfm._stream(None) == 103
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert tfm._stream(None) == 77
    assert tfm._stream(5) == 5 and tfm._stream(types.SimpleNamespace(cuda_stream=6)) == 6
