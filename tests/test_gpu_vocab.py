"""The operators over discrete values (include/tfm_vocab.h) on the GPU against the float64 oracle of
oracle/vocab.py, at the sizes and values where they can go wrong.

Tolerances count roundings.  U = 2^-24 and B = 2^-8 are the largest relative errors of rounding to
float32 and bfloat16.
  embedding forward    the product and the sum round once each, the output once: 2 U (|scale t| +
                       |sum|), and B |value| for a bfloat16 output
  embedding backward   n terms summed in any order: (n + 2) U sum |scale d|
  distillation         with R the largest |s - max| / min(tau, 1) of the row, an exponential is off
                       by at most (4 R + 16) U (its argument has three roundings of size R, and a
                       few ulp of exp), a sum of them by that and the longest chain of additions,
                       V / 64 U: e = (4 R + 32 + V / 64) U each.  Gradients: 2 e times the terms
                       they are made of; row losses: 2 e (2 alpha tau^2 + 1) from the logarithms of
                       the sums, U from the output
  sampling             tokens are equal; log-probabilities U |value| + 1e-9
"""

import math
import sys

import numpy as np
import pytest

from oracle import vocab as ov
from paper_2606_03681_amd import workloads as wl

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    from paper_2606_03681_amd import tfm
    tfm.lib()


def _dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(_torch(dtype))


def _torch(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _host(t):
    return t.double().cpu().numpy()


def _rounded(a, dtype):
    """What a float64 array holds after storage in dtype."""
    return wl.storage_to_f64(wl.to_storage(a, dtype), dtype)


# ---------------------------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------------------------

def _placed(n, stride, E, offset=0):
    """Index array [n0, n1, n2, E] of the rows' elements in a flat buffer, and its length."""
    at = offset + sum(np.arange(n[i]).reshape([-1 if j == i else 1 for j in range(3)]) * stride[i]
                      for i in range(3))
    at = at[..., None] + np.arange(E)
    return at, (int(at.max()) if at.size else 0) + 1 + 5


# n, stride, E, V, offset of the first row: widths on and off the vector sizes, one row, none,
# strides that are no multiple of a vector, axes in another order, rows of a stack input
EMBED = [
    ((1, 1, 1), (0, 0, 1), 1, 1, 0),
    ((1, 1, 7), (0, 0, 3), 3, 2, 1),
    ((1, 1, 0), (0, 0, 8), 8, 5, 0),
    ((1, 1, 65), (0, 0, 64), 64, 10, 0),
    ((1, 1, 300), (0, 0, 33), 32, 7, 0),
    ((1, 1, 257), (0, 0, 192), 192, 1, 0),
    ((3, 5, 4), (5 * 9 * 64, 9 * 64, 64), 64, 31, 64 * 2),
    ((4, 3, 2), (24, 100, 12), 12, 6, 3),        # the middle axis steps farthest
    ((1, 1, 5), (0, 0, 1000), 1000, 50, 0),
    ((1, 1, 9), (0, 0, 2056), 2049, 40, 8),
    ((1, 1, 4096), (0, 0, 40), 40, 3000, 0),
    ((1, 1, 4097), (0, 0, 24), 24, 100003, 0),
    ((2, 500, 20), (500 * 21 * 96, 21 * 96, 96), 96, 37, 0),
]


def _embed_case(n, stride, E, V, offset, rows, table, seed, skew=False):
    rng = np.random.default_rng(seed)
    ids = rng.integers(-2, V + 2, n).astype(np.int32)
    if skew:
        ids[rng.random(n) < 0.7] = V // 2
    at, length = _placed(n, stride, E, offset)
    buf = _rounded(rng.normal(size=length), rows)
    tab = _rounded(rng.normal(size=(V, E)), table)
    return ids, at, buf, tab


def _shape(n, stride, E, V, rows, table, scale):
    from paper_2606_03681_amd import tfm
    return tfm.make_embed(n, stride, E, V, rows, table, scale)


def _buffer(buf, rows, offset):
    """The whole device buffer, and the view that starts at the first row."""
    t = _dev(wl.to_storage(buf, rows))
    if rows == "bf16":
        import torch
        t = t.view(torch.bfloat16)
    return t, t[offset:]


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("table,rows", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"),
                                        ("bf16", "bf16")])
@pytest.mark.parametrize("case", range(len(EMBED)))
def test_embed_fwd(case, table, rows, add):
    import torch
    from paper_2606_03681_amd import tfm
    n, stride, E, V, offset = EMBED[case]
    ids, at, buf, tab = _embed_case(n, stride, E, V, offset, rows, table, case)
    scale = np.float32(1.7)
    whole, out = _buffer(buf, rows, offset)
    tdev = _dev(tab, table)
    tfm.embed_fwd(_shape(n, stride, E, V, rows, table, scale),
                  _dev(ids).reshape(n), tdev, out, add)
    torch.cuda.synchronize()
    got = _host(whole)
    want = buf.copy()
    ref = ov.embed_forward(ids, tab, float(scale), buf[at] if add else None)
    want[at] = ref
    bound = np.zeros_like(buf)
    bound[at] = 2 * U * (np.abs(ov.embed_forward(ids, tab, float(scale))) + np.abs(ref)) + \
        (B if rows == "bf16" else U) * np.abs(ref)
    absent = (ids < 0) | (ids >= V)
    if absent.any():
        bound[at[absent]] = 0                      # zeros, or left exactly as they were
    assert np.all(np.abs(got - want) <= bound)     # elements between the rows included


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("rows", ["f32", "bf16"])
@pytest.mark.parametrize("skew", [False, True])
@pytest.mark.parametrize("case", range(len(EMBED)))
def test_embed_bwd(case, skew, rows, add):
    import torch
    from paper_2606_03681_amd import tfm
    n, stride, E, V, offset = EMBED[case]
    ids, at, buf, _ = _embed_case(n, stride, E, V, offset, rows, "f32", 100 + case, skew)
    scale = np.float32(-0.3)
    e = _shape(n, stride, E, V, rows, "f32", scale)
    whole, dout = _buffer(buf, rows, offset)
    start = np.random.default_rng(9).normal(size=(V, E)).astype(np.float32)
    dtable = _dev(start.copy())
    ws = torch.full((tfm.embed_workspace_bytes(e),), 0xA5, dtype=torch.uint8, device="cuda")
    tfm.embed_bwd(e, _dev(ids).reshape(n), dout, dtable, add, ws)
    torch.cuda.synchronize()
    got = _host(dtable)
    ref = ov.embed_backward(ids, buf[at], V, float(scale))
    count = np.bincount(ids[(ids >= 0) & (ids < V)].ravel(), minlength=V)[:, None]
    bound = (count + 2) * U * ov.embed_backward(ids, np.abs(buf[at]), V, abs(float(scale)))
    if add:
        ref = ref + start
        bound = bound + 2 * U * np.abs(ref) * (count > 0)
    assert np.all(np.abs(got - ref) <= bound)
    again = _dev(start.copy())
    ws.fill_(0x5A)
    tfm.embed_bwd(e, _dev(ids).reshape(n), dout, again, add, ws)
    assert torch.equal(again, dtable)


@pytest.mark.parametrize("rows", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,E,hot", [(20000, 3, 64, 0.9), (70001, 997, 96, 0.5),
                                       (150000, 1, 32, 1.0), (9001, 70000, 136, 0.0)])
def test_embed_bwd_long_runs(N, V, E, hot, rows):
    """Ids that many positions share: sums over thousands of rows, split and joined."""
    import torch
    from paper_2606_03681_amd import tfm
    rng = np.random.default_rng(N)
    ids = rng.integers(0, V, N).astype(np.int32)
    ids[rng.random(N) < hot] = V // 3
    d = _rounded(rng.normal(size=(N, E)), rows)
    e = _shape((1, 1, N), (0, 0, E), E, V, rows, "f32", 1.0)
    dtable = torch.empty((V, E), device="cuda")
    ws = torch.empty(tfm.embed_workspace_bytes(e), dtype=torch.uint8, device="cuda")
    tfm.embed_bwd(e, _dev(ids).reshape(1, 1, N), _dev(d, rows), dtable, False, ws)
    order = np.argsort(ids, kind="stable")
    heads = np.flatnonzero(np.diff(ids[order], prepend=-1))
    ref, mag = np.zeros((V, E)), np.zeros((V, E))
    ref[ids[order][heads]] = np.add.reduceat(d[order], heads, axis=0)
    mag[ids[order][heads]] = np.add.reduceat(np.abs(d[order]), heads, axis=0)
    count = np.bincount(ids, minlength=V)[:, None]
    assert np.all(np.abs(_host(dtable) - ref) <= (count + 2) * U * mag)


def test_embed_bwd_of_a_broadcast_gradient():
    """Rows that all lie on one another, as an expanded gradient has them."""
    import torch
    from paper_2606_03681_amd import tfm
    ids = np.array([[[0, 2, 2, -1, 2]]], np.int32)
    e = _shape((1, 1, 5), (0, 0, 0), 48, 4, "f32", "f32", 2.0)
    d = torch.ones(48, device="cuda")
    dtable = torch.full((4, 48), 9.0, device="cuda")
    ws = torch.empty(tfm.embed_workspace_bytes(e), dtype=torch.uint8, device="cuda")
    tfm.embed_bwd(e, _dev(ids), d, dtable, False, ws)
    assert np.array_equal(_host(dtable), np.outer([2.0, 0.0, 6.0, 0.0], np.ones(48)))


def test_embedding_past_32_bit_offsets():
    import torch
    from paper_2606_03681_amd import tfm
    step, E, V = (1 << 32) + 64, 64, 5
    buf = torch.empty(step + E, dtype=torch.bfloat16, device="cuda")
    buf[:E] = 3.0
    buf[step - 8:] = 3.0
    e = _shape((2, 1, 1), (step, 0, 0), E, V, "bf16", "f32", 1.0)
    ids = _dev(np.array([[[4]], [[1]]], np.int32))
    table = torch.arange(V * E, device="cuda", dtype=torch.float32).reshape(V, E) % 251
    tfm.embed_fwd(e, ids, table, buf)
    assert torch.equal(buf[:E].float(), table[4]) and torch.equal(buf[step:].float(), table[1])
    assert bool((buf[step - 8:step] == 3.0).all())
    dtable = torch.empty((V, E), device="cuda")
    ws = torch.empty(tfm.embed_workspace_bytes(e), dtype=torch.uint8, device="cuda")
    tfm.embed_bwd(e, ids, buf, dtable, False, ws)
    want = torch.zeros_like(table)
    want[4], want[1] = table[4], table[1]
    assert torch.equal(dtable, want)


# ---------------------------------------------------------------------------------------------
# Distillation
# ---------------------------------------------------------------------------------------------

def _logit_rows(z, dtype, pad, offset):
    """Device rows of z, `pad` elements apart and `offset` elements into their buffer, and the
    buffer (its other elements hold 77)."""
    import torch
    N, V = z.shape
    buf = torch.full((offset + N * (V + pad) + 3,), 77.0, dtype=_torch(dtype), device="cuda")
    rows = buf[offset:offset + N * (V + pad)].view(N, V + pad)[:, :V]
    rows.copy_(_dev(z))
    return buf, rows


def _distill_inputs(N, V, k, dtype, seed, spread=3.0, absent=0.1, repeat=0.1):
    rng = np.random.default_rng(seed)
    t = spread * rng.normal(size=(N, V))
    s = _rounded(0.8 * t + 0.5 * rng.normal(size=(N, V)), dtype)
    order = np.argsort(-t, axis=1)[:, :k]
    idx = np.full((N, k), -1, np.int32)
    idx[:, :order.shape[1]] = order
    top = np.where(idx >= 0, np.take_along_axis(t, idx.clip(0), 1), 0.0).astype(np.float32)
    perm = rng.permutation(k)                      # entries in any order
    idx, top = idx[:, perm].copy(), top[:, perm].copy()
    out = rng.random((N, k)) < absent
    idx[out] = rng.choice([-1, V, -2 ** 31, 2 ** 31 - 1], size=int(out.sum()))
    if k > 1:
        rep = rng.random(N) < repeat
        idx[rep, -1] = idx[rep, 0]
    return s, t, idx, top


def _run_distill(s, dtype, idx, top, lse, labels, weights, ncls, tau, alpha, tail, pad=0, offset=0,
                 doffset=None, inplace=False, want_rows=True, want_grad=True):
    import torch
    from paper_2606_03681_amd import tfm
    N, V = s.shape
    d = tfm.make_distill(N, V, idx.shape[1], V + pad, dtype, tau, alpha, tail)
    buf, rows = _logit_rows(s, dtype, pad, offset)
    gbuf, grad = (buf, rows) if inplace else \
        _logit_rows(np.full((N, V), 5.0), dtype, pad, offset if doffset is None else doffset)
    loss = torch.full((2,), 8.0, device="cuda")
    row = torch.full((N,), 8.0, device="cuda") if want_rows else None
    ws = torch.full((tfm.distill_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device="cuda")
    opt = [None if a is None else _dev(a) for a in (lse, labels, weights, ncls)]
    tfm.distill_loss(d, rows, _dev(idx), _dev(top), opt[0], opt[1], opt[2], opt[3], loss, row,
                     grad if want_grad else None, ws)
    torch.cuda.synchronize()
    rest = gbuf.clone()
    goff = offset if doffset is None or inplace else doffset
    if N:
        rest[goff:goff + N * (V + pad)].view(N, V + pad)[:, :V] = 77.0
    assert bool((rest == 77.0).all()), "elements outside the rows were written"
    assert float(loss[1]) == 8.0
    return float(loss[0]), None if row is None else _host(row), _host(grad)


def _check_distill(got, ref, s, labels, weights, ncls, tau, alpha, dtype):
    loss, rows, grad = got
    rloss, rrows, rgrad = ref
    N, V = s.shape
    w = np.ones(N) if weights is None else weights.astype(np.float64)
    live = np.where(np.isfinite(s), s, np.nan)
    if ncls is not None:
        live = np.where(np.arange(V) < ncls[:, None], live, np.nan)
    rtol = np.zeros(N)
    for n in range(N):
        row = live[n][np.isfinite(live[n])]
        R = (row.max() - row.min()) / min(tau, 1.0) if len(row) else 0.0
        e = (4 * R + 32 + V / 64) * U
        rtol[n] = 2 * e * (2 * alpha * tau * tau + 1) + U * abs(rrows[n])
        if not np.isfinite(rrows[n]):
            assert rows is None or rows[n] == rrows[n]
            continue
        if rows is not None:
            assert abs(rows[n] - rrows[n]) <= rtol[n], (n, rows[n], rrows[n], rtol[n])
        # the gradient is a difference of distributions, each at most 1 in every class
        share = abs(w[n]) / w.sum() if w.sum() else 0.0
        q = np.exp((row - row.max()) / tau) if len(row) else np.zeros(1)
        size = np.zeros(V)
        if len(row):
            x = np.where(np.isfinite(live[n]), live[n], -np.inf)
            size = np.exp((x - row.max()) / tau) / q.sum() * alpha * tau * 2
            size = size + (1 - alpha) * np.exp(x - row.max()) / np.exp(row - row.max()).sum()
            # what the teacher adds where it is larger than the student
            size = size + np.abs(rgrad[n]) / (share if share else 1.0)
        bound = 2 * e * share * size + (B if dtype == "bf16" else U) * np.abs(rgrad[n])
        bad = ~(np.abs(grad[n] - rgrad[n]) <= bound + 1e-38)
        assert not bad.any(), (n, np.flatnonzero(bad)[:5], grad[n][bad][:5], rgrad[n][bad][:5])
    if np.isfinite(rloss):
        total = abs(w).sum()
        tol = (np.abs(w) * rtol).sum() / total if total else 0.0
        assert abs(loss - rloss) <= tol + U * abs(rloss), (loss, rloss)
    else:
        assert loss == rloss


DISTILL = [  # N, V, k, pad, offset
    (1, 1, 1, 0, 0), (5, 2, 2, 0, 0), (7, 3, 1, 2, 1), (300, 10, 5, 0, 0), (9, 10, 200, 0, 0),
    (67, 16, 3, 1, 0), (33, 17, 17, 0, 3), (40, 64, 8, 0, 0), (41, 65, 8, 0, 0), (5, 100, 100, 7, 0),
    (6, 255, 33, 0, 0), (6, 256, 256, 0, 0), (17, 1000, 20, 0, 0), (3, 1024, 64, 8, 0),
    (3, 1025, 64, 0, 5), (4, 4099, 32, 0, 1), (3, 5000, 32, 24, 0), (2, 16385, 64, 0, 0),
    (2, 32768, 64, 0, 0), (2, 50021, 64, 1, 0), (1, 131072, 256, 0, 0), (1, 131071, 7, 0, 1),
    (1, 262144, 100, 0, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tail,tau,alpha", [(0, 1.0, 1.0), (1, 2.0, 1.0), (1, 0.7, 0.5),
                                            (0, 3.0, 0.25), (1, 1.0, 0.0)])
@pytest.mark.parametrize("case", range(len(DISTILL)))
def test_distill(case, tail, tau, alpha, dtype):
    N, V, k, pad, offset = DISTILL[case]
    tau, alpha = float(np.float32(tau)), float(np.float32(alpha))
    s, t, idx, top = _distill_inputs(N, V, k, dtype, 1000 + case)
    lse = np.array([ov._logsumexp(row / tau) for row in t]).astype(np.float32) if tail else None
    rng = np.random.default_rng(case)
    labels = rng.integers(-1, V + 1, N).astype(np.int32) if alpha < 1 else None
    weights = None if case % 2 else \
        (rng.random(N) * (rng.random(N) < 0.8)).astype(np.float32)
    ncls = rng.integers(0, V + 2, N).astype(np.int32) if case % 3 == 0 else None
    args = (idx, top, lse, labels, weights, ncls, tau, alpha, tail)
    got = _run_distill(s, dtype, *args, pad=pad, offset=offset, doffset=offset + case % 2,
                       inplace=case % 4 == 3)
    _check_distill(got, ov.distill_loss(s, *args), s, labels, weights, ncls, tau, alpha, dtype)


@pytest.mark.parametrize("V", [3, 12, 64, 200, 3000, 70000])
@pytest.mark.parametrize("tail", [0, 1])
def test_distill_masked_and_empty_rows(tail, V):
    """-inf and lowest-value masks, rows that they leave empty, entries that say nothing, NaN in rows
    of weight 0, labels and entries on masked classes."""
    rng = np.random.default_rng(V)
    N, k, tau = 8, 3, 2.0
    low = np.finfo(np.float32).min
    s = rng.normal(size=(N, V)).astype(np.float32).astype(np.float64)
    idx = np.stack([rng.permutation(V)[:k] for _ in range(N)]).astype(np.int32)
    top = rng.normal(size=(N, k)).astype(np.float32)
    lse = (np.array([ov._logsumexp(r / tau) for r in top]) + 1).astype(np.float32)
    labels = rng.integers(0, V, N).astype(np.int32)
    w = np.ones(N, np.float32)
    s[0] = -np.inf
    s[1, :] = -np.inf
    s[1, idx[1]] = 1.0                      # nothing outside the entries
    s[2, idx[2]] = -np.inf                  # the entries' classes are masked: loss is infinite
    s[3, V // 2:] = low
    s[4] = np.nan
    w[4] = 0.0
    idx[5] = -1
    top[6] = -np.inf
    s[7] = low
    labels[7] = -1
    if V == 3:
        s[2, idx[2, 0]] = 1.0               # (a row of three keeps one class)
    lse = lse if tail else None
    args = (idx, top, lse, labels, w, None, tau, 0.5, tail)
    with np.errstate(invalid="ignore", divide="ignore"):
        ref = ov.distill_loss(s, *args)
    got = _run_distill(s, "f32", *args)
    assert np.isinf(ref[1][2]) and got[1][2] == np.inf
    keep = [0, 1, 3, 4, 5, 6, 7]
    # the finite rows, one by one (the total is infinite as the oracle's is)
    assert got[0] == np.inf == ref[0]
    for n in keep:
        R = 8.0 / 1.0
        e = (4 * R + 32 + V / 64) * U
        # (an entry on a class masked by the lowest value may weigh more than float32 holds)
        if abs(ref[1][n]) > np.finfo(np.float32).max * (1 + U):
            assert got[1][n] == np.inf
            continue
        assert abs(got[1][n] - ref[1][n]) <= 2 * e * (2 * 0.5 * tau * tau + 1) + \
            4 * U * abs(ref[1][n]), n
        assert np.all(np.abs(got[2][n] - ref[2][n]) <= 4 * e / 7 + U * np.abs(ref[2][n])), n
    assert not got[2][0].any() and not got[2][4].any()


def test_distill_values_that_are_not_finite():
    rng = np.random.default_rng(3)
    for V in (10, 100, 5000):
        s = rng.normal(size=(4, V))
        s[0, 1], s[1, 2] = np.nan, np.inf
        idx = np.tile(np.arange(3, dtype=np.int32), (4, 1))
        top = rng.normal(size=(4, 3)).astype(np.float32)
        top[2, 0] = np.nan
        for tail in (0, 1):
            lse = np.full(4, 2.0, np.float32) if tail else None
            loss, rows, grad = _run_distill(s, "f32", idx, top, lse, None, None, None, 1.0, 1.0, tail)
            assert not np.isfinite(rows[:3]).any() and np.isfinite(rows[3])
            ref = ov.distill_row(s[3], idx[3], top[3], 2.0, -1, 1.0, 1.0, tail)
            assert np.abs(grad[3] - ref[1] / 4).max() <= 200 * U


@pytest.mark.parametrize("V,N", [(10, 50), (5000, 9), (60000, 3)])
def test_distill_outputs_one_by_one(V, N):
    """Loss alone, without row losses, and no rows at all give what the whole call gives."""
    import torch
    from paper_2606_03681_amd import tfm
    s, t, idx, top = _distill_inputs(N, V, 6, "bf16", 5)
    lse = np.array([ov._logsumexp(r) for r in t]).astype(np.float32)
    args = (idx, top, lse, None, None, None, 1.0, 1.0, 1)
    full = _run_distill(s, "bf16", *args)
    assert _run_distill(s, "bf16", *args, want_rows=False)[0] == full[0]
    part = _run_distill(s, "bf16", *args, want_grad=False)
    assert part[0] == full[0] and np.array_equal(part[1], full[1])
    assert np.array_equal(_run_distill(s, "bf16", *args, inplace=True)[2], full[2])
    zero = _run_distill(s, "bf16", idx, top, lse, None, np.zeros(N, np.float32), None, 1.0, 1.0, 1)
    assert zero[0] == 0 and not zero[2].any()
    d = tfm.make_distill(0, V, 6, V, "bf16", 1.0, 1.0, 0)
    loss = torch.full((1,), 3.0, device="cuda")
    ws = torch.empty(tfm.distill_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    e = torch.empty((0, V), dtype=torch.bfloat16, device="cuda")
    tfm.distill_loss(d, e, torch.empty((0, 6), dtype=torch.int32, device="cuda"),
                     torch.empty((0, 6), device="cuda"), None, None, None, None, loss, None, e, ws)
    assert float(loss) == 0.0


def test_distill_gradient_against_differences():
    """The kernel's gradient against differences of the kernel's own losses (float32 losses of size
    about 1: steps of 2^-4 leave 2 U / 2^-4 of rounding and h^2 / 6 of curvature, below 1e-3)."""
    V, N, h = 12, 2, 2.0 ** -4
    s, t, idx, top = _distill_inputs(N, V, 4, "f32", 8, spread=1.0, absent=0, repeat=0)
    lse = np.array([ov._logsumexp(r / 2.0) for r in t]).astype(np.float32)
    labels = np.array([3, 7], np.int32)
    args = (idx, top, lse, labels, None, None, 2.0, 0.5, 1)
    _, _, grad = _run_distill(s, "f32", *args)
    for n in range(N):
        for v in range(V):
            d = np.zeros_like(s)
            d[n, v] = h
            up, down = (_run_distill(s + sg * d, "f32", *args)[0] for sg in (1, -1))
            assert abs((up - down) / (2 * h) - grad[n, v]) <= 1e-3


def test_distill_many_rows_and_weights():
    """More rows than one partial sum of the weights holds."""
    import torch
    from paper_2606_03681_amd import tfm
    N, V, k = 40001, 6, 2
    rng = np.random.default_rng(4)
    s, t, idx, top = _distill_inputs(N, V, k, "f32", 12)
    w = rng.random(N).astype(np.float32)
    loss, rows, grad = _run_distill(s, "f32", idx, top, None, None, w, None, 1.0, 1.0, 0)
    total = w.astype(np.float64).sum()
    assert abs(loss - (w * rows).sum() / total) <= 2 * U * abs(loss)
    for n in (0, 1, 4095, 4096, 4097, 20000, 40000):
        L, g = ov.distill_row(s[n], idx[n], top[n], None, -1, 1.0, 1.0, 0)
        assert abs(rows[n] - L) <= 1e3 * U * (abs(L) + 1)
        assert np.abs(grad[n] - g * w[n] / total).max() <= 1e3 * U * w[n] / total


def test_distill_past_32_bit_offsets():
    import torch
    from paper_2606_03681_amd import tfm
    N, V, k, ld = 3, 1000, 4, (1 << 31) + 8
    s, t, idx, top = _distill_inputs(N, V, k, "bf16", 21)
    buf = torch.empty((N - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    rows = buf.as_strided((N, V), (ld, 1))
    rows.copy_(_dev(s))
    d = tfm.make_distill(N, V, k, ld, "bf16")
    loss, row = torch.empty(1, device="cuda"), torch.empty(N, device="cuda")
    ws = torch.empty(tfm.distill_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    u = torch.tensor([0.3, 0.6, 0.9], device="cuda")
    token = torch.empty(N, dtype=torch.int32, device="cuda")
    tfm.sample(tfm.make_sampling(N, V, ld, "bf16"), rows, None, None, None, None, None, u, token)
    tfm.distill_loss(d, rows, _dev(idx), _dev(top), None, None, None, None, loss, row, rows, ws)
    ref = ov.distill_loss(s, idx, top, None, None, None, None, 1.0, 1.0, 0)
    _check_distill((float(loss), _host(row), _host(rows)), ref, s, None, None, None, 1.0, 1.0, "bf16")
    assert token.tolist() == [ov.sample_row(s[n], u=float(u[n]))[0] for n in range(N)]


# ---------------------------------------------------------------------------------------------
# Sampling
# ---------------------------------------------------------------------------------------------

def _run_sample(z, dtype, u, pad=0, offset=0, **kw):
    import torch
    from paper_2606_03681_amd import tfm
    N, V = z.shape
    _, rows = _logit_rows(z, dtype, pad, offset)
    types = dict(n_class=np.int32, temperature=np.float32, top_k=np.int32, top_p=np.float32,
                 min_p=np.float32)
    opt = [None if kw.get(k) is None else _dev(np.asarray(kw[k], ty)) for k, ty in types.items()]
    token = torch.full((N,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((N,), 9.0, device="cuda")
    tfm.sample(tfm.make_sampling(N, V, V + pad, dtype), rows, *opt,
               _dev(np.asarray(u, np.float32)), token, lp)
    torch.cuda.synchronize()
    return token.cpu().numpy(), _host(lp)


def _check_sample(z, dtype, u, pad=0, offset=0, **kw):
    z = _rounded(z, dtype) if np.isfinite(z).all() else z
    token, lp = _run_sample(z, dtype, u, pad, offset, **kw)
    for n in range(len(z)):
        row = z[n]
        set_ = {}
        for k, a in kw.items():
            if a is None:
                continue
            if k == "n_class":
                row = row[:min(max(int(a[n]), 0), z.shape[1])]
            else:
                set_[k] = int(a[n]) if k == "top_k" else float(np.float32(a[n]))
        t, l = ov.sample_row(row, u=float(np.float32(u[n])), **set_)
        assert token[n] == t, (n, token[n], t, set_)
        assert lp[n] == l or abs(lp[n] - l) <= U * abs(l) + 1e-9, (n, lp[n], l)


SIZES = [(1, 1, 0, 0), (40, 2, 0, 0), (30, 3, 1, 1), (200, 10, 0, 0), (20, 16, 0, 0), (21, 17, 3, 0),
         (33, 63, 0, 1), (33, 64, 0, 0), (33, 65, 0, 0), (17, 200, 1, 0), (9, 256, 0, 0),
         (9, 257, 0, 0), (7, 1000, 24, 0), (5, 1024, 0, 0), (5, 1025, 0, 3), (4, 4099, 1, 0),
         (4, 5000, 0, 0), (2, 16385, 0, 0), (2, 32000, 0, 0), (2, 50021, 0, 1), (2, 131072, 0, 0),
         (1, 131071, 1, 0), (1, 262144, 0, 0)]


def _settings(mode, N, V, rng):
    kw = {}
    if mode in ("plain", "mixed"):
        kw["temperature"] = rng.uniform(0.3, 2.0, N)
    if mode in ("k", "kp", "mixed"):
        kw["top_k"] = rng.integers(-1, min(V + 2, 2000), N)
    if mode in ("p", "kp", "mixed"):
        kw["top_p"] = rng.uniform(0.05, 1.05, N)
    if mode in ("min", "mixed"):
        kw["min_p"] = rng.uniform(-0.1, 0.5, N) ** 3
    if mode == "mixed":
        kw["temperature"][rng.random(N) < 0.1] = 0.0
        kw["n_class"] = rng.integers(0, V + 2, N)
    return kw


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["none", "plain", "k", "p", "kp", "min", "mixed"])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_sample(case, mode, dtype):
    N, V, pad, offset = SIZES[case]
    rng = np.random.default_rng(case * 10 + len(mode))
    z = 2.5 * rng.normal(size=(N, V))
    z[:, rng.integers(0, V, 3)] += 4.0
    _check_sample(z, dtype, rng.random(N), pad, offset, **_settings(mode, N, V, rng))


@pytest.mark.parametrize("V", [7, 64, 100, 1500, 5000, 40000, 140000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_ties_and_borders(V, dtype):
    """Few different logits, all equal logits, borders of every rule inside a run of equals, flat and
    very sharp rows."""
    rng = np.random.default_rng(V)
    rows = [np.zeros(V), np.round(rng.normal(size=V)), np.where(np.arange(V) % 3, 1.0, -0.0),
            np.full(V, -88.0), 200.0 * rng.normal(size=V), 1e-3 * rng.normal(size=V),
            np.where(np.arange(V) % 2, 0.0, -0.0)]
    z = np.stack([r for r in rows for _ in range(8)])
    N = len(z)
    kw = dict(top_k=np.tile([0, 1, 2, V // 2, V, V + 5, 3, 0], len(rows)),
              top_p=np.tile([0.5, 1.0, 0.9, 0.25, 1e-6, 0.999, 0.5, 0.75], len(rows)),
              min_p=np.tile([0.0, 0.0, 1.0, 0.0, 0.0, 0.4, 0.3, 0.0], len(rows)))
    u = np.tile([0.0, 0.3, 0.5, 1 - 2.0 ** -24, 0.99, 0.25, 0.75, 0.6], len(rows))
    _check_sample(z, dtype, u, **kw)
    _check_sample(z, dtype, u, top_p=kw["top_p"])
    _check_sample(z, dtype, u, top_k=kw["top_k"], temperature=np.full(N, 1e-3))


@pytest.mark.parametrize("V", [5, 64, 90, 2000, 70000])
def test_sample_values_at_the_edges(V):
    rng = np.random.default_rng(V)
    inf, nan, low = np.inf, np.nan, float(np.finfo(np.float32).min)
    z = rng.normal(size=(12, V)).astype(np.float32).astype(np.float64)
    z[0] = -inf
    z[1] = nan
    z[2, ::2] = -inf
    z[3, 1::2] = nan
    z[4, :2] = inf
    z[5] = low
    z[6, 1:] = low
    z[7] = np.abs(z[7]) * 1e-42               # denormal logits
    z[8, 0] = -low
    z[9, : V - 1] = -inf
    z = z.astype(np.float32).astype(np.float64)   # as stored
    kw = dict(temperature=[1, 1, 1, 1, 1, 1, 1, 1e-40, 1, 1, 1e30, np.nan])
    for u in (0.0, 0.5, 0.999):
        us = np.full(12, u)
        _check_sample(z, "f32", us)
        _check_sample(z, "f32", us, top_p=np.full(12, 0.9), top_k=np.full(12, 3))
        _check_sample(z, "f32", us, **kw)
    _check_sample(z, "f32", np.array([-1.0, 1.0, 2.0, nan, inf, -inf] * 2))
    _check_sample(z, "f32", np.full(12, 0.4), n_class=[0, 1, -3, V, V + 9, 2, 1, 3, 2, V - 1, 4, 5])
    _check_sample(z, "f32", np.full(12, 0.7), top_p=[nan, 0, -1, 2, 0.5, 1, inf, -inf, 0.1, 1, 0, 1],
                  min_p=[nan, 0, -1, 2, 0.5, 1, inf, -inf, 0.1, 1, 0, 1])


def test_sample_row_does_not_depend_on_its_batch():
    rng = np.random.default_rng(2)
    for V in (10, 64, 300, 5000, 60000):
        z = 2 * rng.normal(size=(6, V))
        u = rng.random(6)
        kw = dict(top_p=np.full(6, 0.9), temperature=np.full(6, 0.8))
        token, lp = _run_sample(z, "f32", u, **kw)
        for n in range(6):
            t, l = _run_sample(z[n:n + 1], "f32", u[n:n + 1], offset=n % 4,
                               **{k: a[n:n + 1] for k, a in kw.items()})
            assert t[0] == token[n] and l[0] == lp[n]


def test_sample_draws_follow_the_probabilities():
    """20,000 draws of one row: shares within five standard deviations."""
    rng = np.random.default_rng(11)
    s = 1.5 * rng.normal(size=12)
    N = 20000
    token, _ = _run_sample(np.tile(s, (N, 1)), "f32", rng.random(N), min_p=np.full(N, 0.05))
    p = np.exp(s - s.max())
    p[p < 0.05] = 0
    p /= p.sum()
    share = np.bincount(token, minlength=12) / N
    assert np.all(np.abs(share - p) <= 5 * np.sqrt(p * (1 - p) / N) + 1e-12)


# ---------------------------------------------------------------------------------------------
# Streams and graphs
# ---------------------------------------------------------------------------------------------

def _chain(N=777, V=300, E=64, W=6000):
    """Every operator once on buffers of its own: embedding, its gradient, a distillation over few
    and over many classes, a draw."""
    import torch
    from paper_2606_03681_amd import tfm
    g = torch.Generator(device="cuda").manual_seed(3)
    st = dict(ids=torch.randint(-1, V + 1, (1, 1, N), generator=g, device="cuda").int(),
              table=torch.randn((V, E), generator=g, device="cuda"),
              rows=torch.zeros((N, E), dtype=torch.bfloat16, device="cuda"),
              dtable=torch.zeros((V, E), device="cuda"))
    e = tfm.make_embed((1, 1, N), (0, 0, E), E, V, "bf16", "f32", 0.5)
    st["ews"] = torch.empty(tfm.embed_workspace_bytes(e), dtype=torch.uint8, device="cuda")
    out = ["rows", "dtable"]
    calls = [lambda: tfm.embed_fwd(e, st["ids"], st["table"], st["rows"]),
             lambda: tfm.embed_bwd(e, st["ids"], st["rows"], st["dtable"], False, st["ews"])]
    for tag, M, K, dt in (("a", 200, 10, torch.float32), ("b", 5, W, torch.bfloat16)):
        st["z" + tag] = torch.randn((M, K), generator=g, device="cuda").to(dt)
        st["i" + tag] = torch.randint(0, K, (M, 4), generator=g, device="cuda").int()
        st["t" + tag] = torch.randn((M, 4), generator=g, device="cuda")
        st["w" + tag] = torch.rand(M, generator=g, device="cuda")
        st["u" + tag] = torch.rand(M, generator=g, device="cuda")
        st["d" + tag] = torch.zeros_like(st["z" + tag])
        st["l" + tag] = torch.zeros(1, device="cuda")
        st["k" + tag] = torch.zeros(M, dtype=torch.int32, device="cuda")
        st["p" + tag] = torch.full((M,), 0.8, device="cuda")
        name = "f32" if dt == torch.float32 else "bf16"
        d = tfm.make_distill(M, K, 4, K, name, 1.0, 1.0, 0)
        st["ws" + tag] = torch.empty(tfm.distill_workspace_bytes(d), dtype=torch.uint8,
                                     device="cuda")
        s = tfm.make_sampling(M, K, K, name)
        calls.append(lambda d=d, tag=tag: tfm.distill_loss(
            d, st["z" + tag], st["i" + tag], st["t" + tag], None, None, st["w" + tag], None,
            st["l" + tag], None, st["d" + tag], st["ws" + tag]))
        calls.append(lambda s=s, tag=tag: tfm.sample(
            s, st["z" + tag], None, None, None, st["p" + tag], None, st["u" + tag], st["k" + tag]))
        out += ["d" + tag, "l" + tag, "k" + tag]

    def change(step):
        gg = torch.Generator(device="cuda").manual_seed(100 + step)
        st["ids"].copy_(torch.randint(-1, V + 1, (1, 1, N), generator=gg, device="cuda"))
        for tag in "ab":
            st["z" + tag].copy_(torch.randn(st["z" + tag].shape, generator=gg, device="cuda"))
            st["u" + tag].copy_(torch.rand(st["u" + tag].shape, generator=gg, device="cuda"))

    def run():
        for c in calls:
            c()

    return run, change, lambda: [st[k].clone() for k in out]


def test_operators_on_a_side_stream_and_replayed_from_a_graph():
    import torch
    run, change, outputs = _chain()
    eager = []
    for step in range(4):
        change(step)
        run()
        eager.append(outputs())
    side = torch.cuda.Stream()
    change(1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(outputs(), eager[1]))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for step in (0, 1, 2, 3, 0):
        change(step)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), eager[step])), step
        change(2)                                   # eager work between the replays
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), eager[2]))


def test_operators_on_two_streams_at_once():
    """Two sets of calls with buffers and workspaces of their own, running side by side."""
    import torch
    sets = [_chain(), _chain(N=20001, V=5000, E=64, W=30000)]
    want = []
    for run, change, outputs in sets:
        change(5)
        run()
        want.append(outputs())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(4):
        for s, (run, _, _) in zip(streams, sets):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, _, outputs), ref in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(outputs(), ref))


# ---------------------------------------------------------------------------------------------
# Where one way of working passes into another
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("N", [0, 1, 16384, 16385, 100003, 2200000])
@pytest.mark.parametrize("weighted", [False, True])
def test_distill_total_over_few_and_many_rows(N, weighted):
    """The loss is the 64-bit weighted mean of the rows' own losses, rounded once."""
    import torch
    from paper_2606_03681_amd import tfm
    V, k = 3, 2
    g = torch.Generator(device="cuda").manual_seed(N + weighted)
    z = torch.randn((N, V), generator=g, device="cuda")
    idx = torch.randint(0, V, (N, k), generator=g, device="cuda").int()
    top = torch.randn((N, k), generator=g, device="cuda")
    w = torch.rand(N, generator=g, device="cuda") if weighted else None
    if weighted:
        w[::7] = 0
    d = tfm.make_distill(N, V, k, V, "f32", 1.0, 1.0, 0)
    ws = torch.full((tfm.distill_workspace_bytes(d),), 0xA5, dtype=torch.uint8, device="cuda")
    rows, loss = torch.empty(N, device="cuda"), torch.empty(2, device="cuda")
    tfm.distill_loss(d, z, idx, top, None, None, w, None, loss, rows, None, ws)
    tfm.distill_loss(d, z, idx, top, None, None, w, None, loss[1:], None, None, ws)
    wd = torch.ones(N, dtype=torch.float64) if w is None else w.double().cpu()
    total = float(wd.sum())
    ref = float((wd * rows.double().cpu()).sum()) / total if total else 0.0
    assert abs(float(loss[0]) - ref) <= 2 * U * abs(ref)      # one rounding, and the reference's own
    assert float(loss[1]) == float(loss[0])                   # rows in the workspace: the same
    for n in {0, N // 2, N - 1} if N else ():
        L, _ = ov.distill_row(z[n].double().cpu().numpy(), idx[n].cpu().numpy(),
                              top[n].cpu().numpy(), None, -1, 1.0, 1.0, 0)
        L = 0.0 if wd[n] == 0 else L
        assert abs(float(rows[n]) - L) <= 1e3 * U * (abs(L) + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(64, 24575), (64, 24576), (65, 24576), (63, 24584), (64, 33001)])
@pytest.mark.parametrize("tail,tau,alpha", [(0, 1.0, 1.0), (1, 3.0, 0.25)])
def test_distill_around_split_rows(N, V, tail, tau, alpha, dtype):
    s, t, idx, top = _distill_inputs(N, V, 16, dtype, N + V)
    rng = np.random.default_rng(N * V)
    lse = np.array([ov._logsumexp(r / tau) for r in t]).astype(np.float32) if tail else None
    labels = rng.integers(-1, V, N).astype(np.int32)
    w = (rng.random(N) < 0.9).astype(np.float32) * rng.uniform(0.5, 2.0, N).astype(np.float32)
    ncls = rng.integers(V // 2, V + 1, N).astype(np.int32)
    args = (idx, top, lse, labels, w, ncls, tau, alpha, tail)
    _check_distill(_run_distill(s, dtype, *args), ov.distill_loss(s, *args), s, labels, w, ncls, tau,
                   alpha, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2049, 5000, 9001, 33000])
def test_sample_row_is_the_same_in_few_and_many_rows(V, dtype):
    """Few long rows and many of them run in workgroups of different sizes."""
    import torch
    from paper_2606_03681_amd import tfm
    N = 1100
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (3 * torch.randn((N, V), generator=g, device="cuda")).to(_torch(dtype))
    u = torch.rand(N, generator=g, device="cuda")
    t = 0.5 + torch.rand(N, generator=g, device="cuda")
    k = torch.randint(0, 300, (N,), generator=g, device="cuda").int()
    p = 0.5 + 0.6 * torch.rand(N, generator=g, device="cuda")
    m = 0.02 * torch.rand(N, generator=g, device="cuda")

    def draw(a, b):
        n = b - a
        token = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        lp = torch.empty(n, device="cuda")
        tfm.sample(tfm.make_sampling(n, V, V, dtype), z[a:b], None, t[a:b], k[a:b], p[a:b], m[a:b],
                   u[a:b], token, lp)
        return token, lp

    token, lp = draw(0, N)
    assert bool((token >= 0).all())
    for a, b in ((0, 1), (1, 513), (513, 1025), (1025, N)):
        tt, ll = draw(a, b)
        assert torch.equal(tt, token[a:b]) and torch.equal(ll, lp[a:b])


@pytest.mark.parametrize("V", [5, 64, 90, 1500, 5000, 70000])
def test_sample_min_p_next_to_zero(V):
    """Borders top + log(min_p) temperature that cancel to about 0, where float32 keys are densest:
    the logits lie on both sides of the border, at least a thousandth of the largest away from it."""
    top = [float.fromhex("0x1.485ff2p+0"), 2.384186e-07, math.log(10.0), 2 * math.log(4.0)]
    tau = [float.fromhex("0x1.1d3904p-1"), 1.0, 1.0, 2.0]
    min_p = [0.1, 0.99999976, 0.1, 0.25]
    shares = np.array([1.0, 0.25, -0.25, 1e-3, -1e-3])
    z = np.stack([t * shares[np.arange(V) % 5] for t in top for _ in range(4)])
    z = z.astype(np.float32).astype(np.float64)
    N = len(z)
    u = np.random.default_rng(V).random(N)
    kw = dict(temperature=np.repeat(tau, 4), min_p=np.repeat(min_p, 4))
    _check_sample(z, "f32", u, **kw)
    _check_sample(z, "f32", u, top_k=np.full(N, 4 * V // 5), **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [3, 12, 64, 200, 1024, 3000, 70000])
@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("alpha,tau", [(1.0, 1.0), (0.5, 2.0), (0.0, 1.0)])
def test_distill_rows_of_nan(tail, V, dtype, alpha, tau):
    """A logit that is NaN shows in the row's loss where nothing lies above -inf, and where the NaN
    stands on an entry without weight; rows of -inf beside them are left out, the rest keeps its
    values.  Split rows, whole ones, unaligned gradients and short rows."""
    nan, inf = np.nan, np.inf
    rng = np.random.default_rng(V + tail)
    N, k = 8, 2
    s = _rounded(rng.normal(size=(N, V)), dtype)
    idx = np.stack([rng.permutation(V)[:k] for _ in range(N)]).astype(np.int32)
    top = rng.normal(size=(N, k)).astype(np.float32)
    lse = np.array([ov._logsumexp(r / tau) + 1 for r in top]).astype(np.float32) if tail else None
    labels = idx[:, 0].copy()
    s[0] = nan
    s[1] = -inf
    s[1, idx[1, 0]] = nan                          # on an entry and the label
    s[2] = -inf
    s[2, (set(range(V)) - set(idx[2].tolist())).pop()] = nan   # outside the entries
    s[3] = -inf                                    # left out
    s[4, idx[4, 1]] = nan                          # on an entry that weighs nothing
    top[4, 1] = -inf
    s[5, idx[5]] = nan                             # on all entries, which weigh nothing
    top[5] = -inf
    ncls = np.full(N, V, np.int32)
    s[6] = nan
    ncls[6] = 0                                    # no class: left out
    args = (idx, top, lse, labels if alpha < 1 else None, None, ncls, tau, alpha, tail)
    ref = ov.distill_loss(s[[3, 6, 7]], *[a[[3, 6, 7]] if isinstance(a, np.ndarray) else a
                                         for a in args])
    for kw in (dict(), dict(doffset=1), dict(inplace=True), dict(pad=1)):
        loss, rows, grad = _run_distill(s, dtype, *args, **kw)
        assert np.isnan(loss)
        for n in (0, 1, 2, 4, 5):
            assert np.isnan(rows[n]) and np.isnan(grad[n]).any(), (n, rows[n])
        for n in (3, 6):
            assert rows[n] == 0 and not grad[n].any(), n
        R = (s[7].max() - s[7].min()) / min(tau, 1.0)
        e = (4 * R + 32 + V / 64) * U
        assert abs(rows[7] - ref[1][2]) <= 2 * e * (2 * alpha * tau * tau + 1) + U * abs(ref[1][2])
        want = ref[2][2] * 3 / N
        # terms of at most 1 in every class, as alpha tau times two distributions and two more
        assert np.all(np.abs(grad[7] - want) <= 2 * e * (2 * alpha * tau + 2) / N +
                      (B if dtype == "bf16" else U) * np.abs(want))


@pytest.mark.parametrize("rows", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,E", [(30001, 997, 192), (20000, 3, 64), (5000, 700, 100),
                                   (9001, 300, 33), (3000, 50, 1032)])
@pytest.mark.parametrize("add", [False, True])
def test_embed_bwd_is_the_same_wherever_the_rows_lie(N, V, E, rows, add):
    """Rows and a gradient on smaller boundaries than a vector's, and rows farther apart: the sums
    keep their order, so the gradient is the same bit for bit."""
    import torch
    from paper_2606_03681_amd import tfm
    g = torch.Generator(device="cuda").manual_seed(N)
    ids = torch.randint(-1, V, (1, 1, N), generator=g, device="cuda").int()
    ids[torch.rand(ids.shape, generator=g, device="cuda") < 0.4] = V // 2
    src = torch.randn((N, E), generator=g, device="cuda").to(_torch(rows))
    start = torch.randn((V, E), generator=g, device="cuda")
    want = None
    for pad, offset, at in ((0, 0, 0), (8, 0, 0), (4, 4, 2), (2, 2, 1), (1, 1, 3), (7, 3, 0), (0, 1, 1)):
        buf = torch.zeros(offset + N * (E + pad) + 8, dtype=_torch(rows), device="cuda")
        buf[offset:offset + N * (E + pad)].view(N, E + pad)[:, :E] = src
        e = _shape((1, 1, N), (0, 0, E + pad), E, V, rows, "f32", 0.7)
        whole = torch.full((at + V * E + 5,), 77.0, device="cuda")
        dtable = whole[at:at + V * E].view(V, E)
        dtable.copy_(start)
        ws = torch.full((tfm.embed_workspace_bytes(e),), 0xA5, dtype=torch.uint8, device="cuda")
        tfm.embed_bwd(e, ids, buf[offset:], dtable, add, ws)
        want = dtable.clone() if want is None else want
        assert torch.equal(dtable, want), (pad, offset, at)
        assert bool((whole[:at] == 77.0).all()) and bool((whole[at + V * E:] == 77.0).all())


def test_missing_workspaces_refused():
    import torch
    from paper_2606_03681_amd import tfm
    ids = torch.zeros((1, 1, 4), dtype=torch.int32, device="cuda")
    rows, table = torch.zeros((4, 32), device="cuda"), torch.zeros((10, 32), device="cuda")
    with pytest.raises(tfm.TfmError, match="workspace"):
        tfm.embed_bwd(_shape((1, 1, 4), (0, 0, 32), 32, 10, "f32", "f32", 1.0), ids, rows, table,
                      False, None)
    z, one = torch.zeros((2, 8), device="cuda"), torch.zeros((2, 1), device="cuda")
    with pytest.raises(tfm.TfmError, match="workspace"):
        tfm.distill_loss(tfm.make_distill(2, 8, 1, 8, "f32"), z, one.int(), one, None, None, None,
                         None, torch.zeros(1, device="cuda"), None, z, None)


def test_sample_top_p_next_to_one_over_a_flat_tail():
    """Two heavy classes and 262,142 light ones of 4.53 steps of 2^-44 each, which round to 5, while
    top_p = 1 - 2^-24 leaves out 4.6 steps per class: by either count the last heavy class is drawn
    where u reaches it, and no light one although all of them together may not be left out."""
    V = 1 << 18
    z = np.full((2, V), np.log(4.53) - 44 * np.log(2.0))
    z[:, 0], z[:, 4096] = 0.0, np.log(0.15)       # (of two threads)
    z = z.astype(np.float32).astype(np.float64)
    p = np.full(2, 1 - 2.0 ** -24)
    _check_sample(z, "f32", np.array([1 - 2.0 ** -24, 0.5]), top_p=p)
