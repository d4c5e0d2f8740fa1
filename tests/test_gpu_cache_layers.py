"""The 8-bit caches inside the framework's own path: context and query calls of the layers
(tfm_layer_fwd_context8, tfm_layer_fwd_query8), stack.InferStack and stack.InferModel with cache8, and
draws from adjusted logits.

The query call against an 8-bit cache is the bfloat16 query call against the values that the cache
stands for (three bits of fraction: exact as bfloat16): outputs agree to the layers' bfloat16
tolerance, and with the oracle's attention over those values to the attention's own bounds."""

import sys

import numpy as np
import pytest

from oracle import cache as oc
from oracle import vocab as ov
from paper_2606_03681_amd import workloads as wl

from _harness import TOL, ends_dims, ends_setup, ends_struct, nerr, storage_of, to_dev

pytestmark = pytest.mark.gpu


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    from paper_2606_03681_amd import tfm
    tfm.lib()


def _dims(w, R):
    from paper_2606_03681_amd import tfm
    kw = {k: v for k, v in w.dims.items() if k not in ("dtype", "R")}
    return tfm.make_dims(dtype=w.dtype, block=w.block, R=R, **kw)


def _setup(name):
    from paper_2606_03681_amd.stack import to_device
    w = wl.make_workload(name)
    R = w.cfg["R"]
    Rc = R - (R // 3 + 5)
    n_train = np.minimum(w.n_train, Rc).astype(np.int32)
    return w, R, Rc, n_train, to_device(np.ascontiguousarray(w.X[:, :Rc]), "bf16")


def _half(w, Rc):
    """Bytes of the keys of a bfloat16 cache, and its active columns' shape."""
    d = w.dims
    B, S = len(w.n_train), d["C"] + 1
    return (B * S * Rc * d["E"] * 2 + 255) // 256 * 256


NAMES = ["ragged-small-bf16", "d16-bf16", "d64-bf16", "prenorm-small-bf16", "prenorm-d64-bf16"]


@pytest.mark.parametrize("name", NAMES)
def test_context_keeps_its_rows_in_8_bits(name):
    """The context call's outputs do not change, and the pool is what appending the bfloat16 keys and
    values gives, page by page; the rest of it is left as it was."""
    import torch
    from paper_2606_03681_amd import tfm
    from paper_2606_03681_amd.stack import InferStack
    w, R, Rc, n_train, X = _setup(name)
    d, dims = w.dims, _dims(w, Rc)
    one = w.params[:1]
    a = InferStack(dims, n_train, w.cell_mask, one, max_query_rows=8)
    b = InferStack(dims, n_train, w.cell_mask, one, max_query_rows=8, cache8=True)
    b.caches[0].fill_(0x55)
    assert torch.equal(a.context(X), b.context(X))
    H, hd = d["heads"], d["E"] // d["heads"]
    ppc = -(-Rc // 64)
    n_pages = len(w.n_train) * (d["C"] + 1) * ppc
    c = tfm.make_cache8(H, hd, 64, n_pages)
    assert b.caches[0].numel() == tfm.cache8_bytes(c) == tfm.infer_cache8_bytes(dims)
    ntr = np.concatenate([np.full(int(m.sum()), n) for m, n in zip(w.cell_mask, n_train)])
    A, half = len(ntr), _half(w, Rc)
    kv = [storage_of(t[:A * H * Rc * hd * 2].view(torch.bfloat16), "bf16")
          for t in (a.caches[0][:half], a.caches[0][half:])]
    k, v = (wl.storage_to_f64(t, "bf16").reshape(A, H, Rc, hd).transpose(0, 2, 1, 3) for t in kv)
    got = [t.view(torch.uint8).cpu().numpy() for t in tfm.cache8_views(c, b.caches[0])]
    for col in range(A):                      # every column, a few of them against the oracle
        if col % max(1, A // 6) and col != A - 1:
            continue
        at = slice(col * ppc, (col + 1) * ppc)
        blank = tuple(np.full_like(g[at], 0x55) for g in got)
        want = oc.append(*blank, k[col:col + 1], v[col:col + 1], ppc, None, None, [ntr[col]])
        for x, y in zip(got, want):
            assert np.array_equal(x[at], y), col
    for x in got:
        assert np.all(x[A * ppc:] == 0x55)


def _as_bf16(w, Rc, n_train, dims, pool):
    """A bfloat16 cache of the values that the pool's rows stand for."""
    import torch
    from paper_2606_03681_amd import tfm
    d = w.dims
    H, hd, ppc = d["heads"], d["E"] // d["heads"], -(-Rc // 64)
    n_pages = len(w.n_train) * (d["C"] + 1) * ppc
    keys, values, powers = tfm.cache8_views(tfm.make_cache8(H, hd, 64, n_pages), pool)
    A, half = int(w.cell_mask.sum()), _half(w, Rc)
    cache = torch.zeros(tfm.infer_cache_bytes(dims), dtype=torch.uint8, device="cuda")
    two = torch.exp2(powers[:A * ppc].float() - 127)
    ntr = np.concatenate([np.full(int(m.sum()), n) for m, n in zip(w.cell_mask, n_train)])
    held = torch.arange(Rc, device="cuda")[None] < to_dev(ntr)[:, None]
    for at, x in ((0, keys[:A * ppc].float() * two[:, :, 0, None, None]),
                  (half, values[:A * ppc].float().transpose(2, 3) * two[:, :, 1, None, None])):
        rows = x.reshape(A, ppc, H, 64, hd).transpose(1, 2).reshape(A, H, ppc * 64, hd)[:, :, :Rc]
        to = cache[at:at + A * H * Rc * hd * 2].view(torch.bfloat16).view(A, H, Rc, hd)
        rows = torch.where(held[:, None, :, None], rows, 0.0)
        to.copy_(rows)
        assert bool((to.float() == rows).all())                # exact
    return cache


@pytest.mark.parametrize("name", NAMES)
def test_query_reads_the_8_bit_cache(name):
    import torch
    from paper_2606_03681_amd import tfm
    from paper_2606_03681_amd.stack import InferStack, to_device
    w, R, Rc, n_train, X = _setup(name)
    dims = _dims(w, Rc)
    st = InferStack(dims, n_train, w.cell_mask, w.params[:1], max_query_rows=R - Rc, cache8=True)
    st.context(X)
    cache = _as_bf16(w, Rc, n_train, dims, st.caches[0])
    for a, b in ((Rc, R), (Rc, Rc + 1), (Rc + 3, Rc + 40)):
        xq = to_device(np.ascontiguousarray(w.X[:, a:b]), "bf16")
        got = st.query(xq).clone()
        want = torch.empty_like(got)
        tfm.layer_fwd_query(_dims(w, b - a), Rc, n_train, w.cell_mask, xq, st.params[0], cache, want,
                            st.workspace)
        e = nerr(wl.storage_to_f64(storage_of(got, "bf16"), "bf16"),
                 wl.storage_to_f64(storage_of(want, "bf16"), "bf16"))
        _say(f"[cache8] {name} rows {a}..{b}: {e:.3g}")
        assert e <= TOL["bf16"]
        st.workspace.fill_(0xFF)                               # nothing kept between calls
        assert torch.equal(st.query(xq), got)


def test_long_context_of_few_columns_is_split():
    """Scratch of a call whose keys are split over workgroups: sized by dims, enough for any mask."""
    import torch
    from paper_2606_03681_amd import tfm
    from paper_2606_03681_amd.stack import to_device
    rng = np.random.default_rng(0)
    B, C, Rc, E, H, heads = 1, 3, 4000, 64, 64, 2
    mk = lambda R: tfm.make_dims(B, R, C, E, heads, H, "bf16")  # noqa: E731
    assert tfm.infer8_workspace_bytes(mk(5), Rc) > tfm.infer_workspace_bytes(mk(5))
    mask = np.array([[1, 0, 0, 1]], np.uint8)
    n_train = np.array([3777], np.int32)
    params = torch.from_numpy(rng.normal(0, 0.08, tfm.param_count(mk(5))).astype(np.float32)).cuda()
    X = to_device(wl.to_storage(rng.normal(size=(B, Rc, C + 1, E)), "bf16"), "bf16")
    xq = to_device(wl.to_storage(rng.normal(size=(B, 5, C + 1, E)), "bf16"), "bf16")
    ws = torch.full((max(tfm.infer_workspace_bytes(mk(Rc)), tfm.infer8_workspace_bytes(mk(5), Rc)),),
                    0xFF, dtype=torch.uint8, device="cuda")
    kv = torch.zeros(tfm.infer_cache_bytes(mk(Rc)), dtype=torch.uint8, device="cuda")
    pool = torch.zeros(tfm.infer_cache8_bytes(mk(Rc)), dtype=torch.uint8, device="cuda")
    Y, Yq, ref = torch.empty_like(X), torch.empty_like(xq), torch.empty_like(xq)
    tfm.layer_fwd_context8(mk(Rc), n_train, mask, X, params, Y, kv, pool, ws)
    need = tfm.infer8_workspace_bytes(mk(5), Rc)
    tfm.layer_fwd_query8(mk(5), Rc, n_train, mask, xq, params, pool, Yq, ws[:need])
    tfm.layer_fwd_query(mk(5), Rc, n_train, mask, xq, params, kv, ref, ws)
    # keys and values differ by up to 2^-4 of each; an average over some 3,777 rows by far less
    e = nerr(Yq.double().cpu().numpy(), ref.double().cpu().numpy())
    _say(f"[cache8] long context against the bfloat16 cache: {e:.3g}")
    assert e <= 2.0 ** -4
    assert bool((Yq[:, :, 1:3] == 0).all())
    with pytest.raises(tfm.TfmError, match="workspace"):
        tfm.layer_fwd_query8(mk(5), Rc, n_train, mask, xq, params, pool, Yq, ws[:need - 1])


@pytest.mark.parametrize("name,T", [("d16-bf16", 0), ("prenorm-small-bf16", 4)])
def test_evaluation_with_8_bit_caches_and_adjusted_draws(name, T):
    import torch
    from paper_2606_03681_amd.stack import InferModel
    w, e = ends_setup(name, T=T)
    dims, en = ends_dims(w), ends_struct(e)
    x, lab = to_dev(e.x), to_dev(e.labels)
    args = (dims, en, w.n_train, e.n_feat, w.params, e.params, e.table)
    im, ref = InferModel(*args, chunk=16, cache8=True), InferModel(*args, chunk=16)
    d = w.dims               # a byte a value in whole pages, and two for each page and head
    assert im.stack.caches[0].numel() == len(w.n_train) * (d["C"] + 1) * -(-im.Rc // 64) * \
        (2 * 64 * d["E"] + 2 * d["heads"])
    z, z0 = im.predict(x, lab), ref.predict(x, lab)
    # the context call's unlabelled rows see no cache: the same bits
    rows, at, ctx = w.cfg["R"] - w.n_train, 0, im.Rc - w.n_train
    for n, k in zip(rows, ctx):
        assert torch.equal(z[at:at + k], z0[at:at + k])
        at += int(n)
    assert torch.isfinite(z).all() and torch.equal(z, im.predict(x, lab))
    rng = np.random.default_rng(4)
    N, K = z.shape
    u = rng.random(N).astype(np.float32)
    bias = rng.normal(size=(N, K)).astype(np.float32)
    allowed = rng.random((N, K)) < 0.7
    hist = rng.integers(-1, K, (N, 5)).astype(np.int32)
    nc = np.repeat(e.n_class, rows)
    token, lp, adj = im.draw(x, lab, to_dev(u), n_class=e.n_class, adjust=dict(
        bias=to_dev(bias), allowed=to_dev(allowed), history=to_dev(hist), n_history=4,
        repetition=1.5, presence=0.25, frequency=0.125))
    zh, ah = z.double().cpu().numpy(), adj.double().cpu().numpy()
    for n in range(N):
        words = [sum(int(allowed[n, i]) << (i - 32 * j) for i in range(32 * j, min(K, 32 * j + 32)))
                 for j in range(-(-K // 32))]
        want, size = ov.adjust_row(zh[n], nc[n], hist[n, :4], 1.5, 0.25, 0.125, range(K), bias[n], words)
        ok = want > -np.inf
        assert np.array_equal(ah[n] > -np.inf, ok)
        assert np.all(np.abs(ah[n] - np.where(ok, want, 0))[ok] <= 1.01 * 2.0 ** -24 * size[ok])
        t, l = ov.sample_row(ah[n, :nc[n]], u=float(u[n]))
        assert int(token[n]) == t
    # one bias and mask for all rows, and a mask that leaves nothing
    _, _, adj = im.draw(x, lab, to_dev(u), adjust=dict(bias=to_dev(bias[0]),
                                                       allowed=to_dev(np.zeros(K, bool))))
    assert bool((adj == -float("inf")).all())
    token, _, _ = im.draw(x, lab, to_dev(u), adjust=dict(allowed=to_dev(np.arange(K) == K - 1)))
    assert bool((token == K - 1).all())
