"""The operators over discrete values inside the framework's own paths: a training step with
categorical columns and a teacher (stack.TrainStep), the decoder's backward for a given gradient,
draws from the forward-only path (stack.InferModel), against the float64 oracles put together.
Tolerances: the ends' (1e-4 float32, 2e-2 bfloat16, normwise)."""

import sys

import numpy as np
import pytest

import oracle
from oracle import ends as oe
from oracle import vocab as ov
from paper_2606_03681_amd import workloads as wl
from paper_2606_03681_amd.stack import to_device

from _harness import (TOL, ends_dims, ends_oracle_params, ends_setup, ends_struct, full_labels,
                      nerr, oracle_encode, oracle_params, to_dev)

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


def _cats(w, e, cols, V, seed):
    """Ids of the first columns (absent ones among them) and their table; x is 0 there."""
    rng = np.random.default_rng(seed)
    B, R, E = len(w.n_train), w.cfg["R"], w.cfg["E"]
    ids = rng.integers(-1, V, (B, R - e.T, cols)).astype(np.int32)
    e.x[:, :, :cols] = 0.0
    return ids, rng.normal(0, 0.5, (V, E)).astype(np.float32)


def _teacher(w, e, k, tau, seed):
    rng = np.random.default_rng(seed)
    rows = w.cfg["R"] - w.n_train
    N = int(rows.sum())
    nc = np.repeat(e.n_class, rows)
    t = 2 * rng.normal(size=(N, e.K))
    t[np.arange(e.K) >= nc[:, None]] = -np.inf
    order = np.argsort(-t, axis=1)[:, :k]
    top = np.take_along_axis(t, order, 1)
    idx = np.where(np.isfinite(top), order, -1).astype(np.int32)
    lse = np.array([ov._logsumexp(r / tau) for r in t]).astype(np.float32)
    return nc.astype(np.int32), idx, np.where(idx >= 0, top, 0).astype(np.float32), lse


STEPS = [("d64-f32", 0, False, 0, 1.0), ("ragged-small-f32", 2, True, 1, 0.5),
         ("prenorm-small-bf16", 4, True, 1, 0.5), ("d16-bf16", 0, False, 0, 0.5)]


@pytest.mark.parametrize("name,T,mean,tail,alpha", STEPS)
def test_training_step_with_categories_and_teacher(name, T, mean, tail, alpha):
    import torch
    from paper_2606_03681_amd.stack import OPTIM_BASELINE, Optimizer, TrainStep
    w, e = ends_setup(name, T=T, mean=mean)
    cols, V, k, tau, scale = min(3, w.cfg["C"]), 11, 4, 2.0, 1.5
    ids, table = _cats(w, e, cols, V, 1)
    nc, idx, top, lse = _teacher(w, e, k, tau, 2)
    C, heads = w.cfg["C"], w.cfg["heads"]
    mode = "mean" if e.mean else "target"
    # the oracles put together
    P = ends_oracle_params(w, e)
    Xd, _, cache = oracle_encode(w, e)
    Xd[:, :, :cols] += ov.embed_forward(ids, table, scale)
    X = oracle.thinking_rows_forward(Xd, e.table.astype(np.float64), e.cell_mask) if T else Xd
    if w.block == "pre":
        Y, caches = oracle.prenorm_stack_forward(X, oracle_params(w), w.n_train, e.cell_mask, heads)
    else:
        Y, caches = oracle.stack_forward(X, oracle_params(w), w.n_train, e.cell_mask, heads)
    z = oe.decode_logits(Y, w.n_train, e.n_feat, C, P, mode)
    y = full_labels(w, e)
    lab = np.concatenate([y[b][int(n):] for b, n in enumerate(w.n_train)]).astype(np.int32)
    rl, _, dlog = ov.distill_loss(z, idx, top, lse, lab if alpha < 1 else None, None, nc, tau, alpha,
                                  tail)
    dY, dP = oe.decode_backward(Y, w.n_train, e.n_feat, C, P, mode, dlog)
    dX, grads = (oracle.prenorm_stack_backward if w.block == "pre" else
                 oracle.stack_backward)(dY, caches)
    dX, dtable = oracle.thinking_rows_backward(dX, e.cell_mask, T) if T else (dX, None)
    dP.update(oe.encode_backward(dX, cache))
    active = e.cell_mask[:, None, :cols] != 0
    dcat = ov.embed_backward(np.where(active, ids, -1), dX[:, :, :cols], V, scale)
    # the framework's step
    ts = TrainStep(ends_dims(w), ends_struct(e), w.n_train, e.n_feat, e.n_class, w.params, e.params,
                   e.table, cat_table=table, cat_cols=cols, cat_scale=scale,
                   distill=dict(k=k, temperature=tau, alpha=alpha, tail=tail))
    teacher = (to_dev(idx), to_dev(top)) + ((to_dev(lse),) if tail else ())
    x, labels = to_dev(e.x), to_dev(e.labels)
    loss = float(ts.run(x, labels, cat_ids=to_dev(ids), teacher=teacher).item())
    tol = TOL[w.dtype]
    _say(f"[vocab-step] {name}: loss {loss:.6g} vs {rl:.6g}")
    assert abs(loss - rl) <= tol * abs(rl)
    got = oe.unpack_ends_params(ts.ends_grads.double().cpu().numpy(), w.cfg["E"], e.G, e.Hd, e.K)
    errs = {n: nerr(got[n], dP[n]) for n in oe.ENDS_PARAM_ORDER}
    errs["cat_table"] = nerr(ts.cat_grad.double().cpu().numpy(), dcat)
    if T:
        errs["thinking"] = nerr(ts.table_grad.double().cpu().numpy(), dtable)
    E, H = w.cfg["E"], w.cfg["H"]
    unpack = oracle.unpack_prenorm_params if w.block == "pre" else oracle.unpack_params
    pack = oracle.pack_prenorm_params if w.block == "pre" else oracle.pack_params
    for l, (gg, gr) in enumerate(zip(ts.stack.grads, grads)):
        pg, pr = unpack(gg.double().cpu().numpy(), E, H), unpack(pack(gr), E, H)
        errs.update({f"L{l}.{n}": nerr(pg[n], pr[n]) for n in pr})
    _say(f"[vocab-step] {name}: worst {max(errs.items(), key=lambda i: i[1])}")
    assert all(v <= tol for v in errs.values()), errs
    # the optimiser owns the table too
    before = ts.cat_table.clone()
    Optimizer(ts, OPTIM_BASELINE).step()
    moved = (ts.cat_table - before).abs().amax(1)
    assert bool(((moved > 0) == (ts.cat_grad.abs().amax(1) > 0)).all()) and bool((moved > 0).any())
    with pytest.raises(ValueError):
        ts.run(x, labels)


DEC = [("ragged-small-f32", 0, False), ("ragged-small-bf16", 0, True),
       ("prenorm-small-bf16", 5, True)]


@pytest.mark.parametrize("name,T,mean", DEC)
def test_decode_bwd_against_oracle(name, T, mean):
    import torch
    from paper_2606_03681_amd import tfm
    w, e = ends_setup(name, T=T, mean=mean)
    w.n_train[0] = w.cfg["R"]              # a dataset without unlabelled rows
    w.n_train[1] = 0                       # and one without labelled ones
    dt, R, C, E = w.dtype, w.cfg["R"], w.cfg["C"], w.cfg["E"]
    B = len(w.n_train)
    rng = np.random.default_rng(4)
    Ys = wl.to_storage(rng.normal(size=(B, R, C + 1, E)), dt)
    N = int((R - w.n_train).sum())
    dlog = rng.normal(size=(N, e.K)).astype(np.float32)
    dims, en = ends_dims(w), ends_struct(e)
    ws = torch.empty(tfm.ends_workspace_bytes(dims, en), dtype=torch.uint8, device="cuda")
    Y = to_device(Ys, dt)
    dY = torch.full_like(Y, 5.0)
    grads = torch.full((len(e.params),), 7.0, device="cuda")
    args = (dims, en, w.n_train, e.n_feat, Y, to_dev(e.params), to_dev(dlog))
    tfm.decode_bwd(*args, dY, grads, False, ws)
    P = ends_oracle_params(w, e)
    rY, rP = oe.decode_backward(wl.storage_to_f64(Ys, dt), w.n_train, e.n_feat, C, P,
                                "mean" if e.mean else "target", dlog.astype(np.float64))
    assert nerr(dY.double().cpu().numpy(), rY) <= TOL[dt]
    g = grads.double().cpu().numpy()
    got = oe.unpack_ends_params(g, E, e.G, e.Hd, e.K)
    for n in ("W_d1", "b_d1", "W_d2", "b_d2"):
        assert nerr(got[n], rP[n]) <= TOL[dt], n
    enc = E * e.G + 3 * E
    assert np.all(g[:enc] == 7.0)
    tfm.decode_bwd(*args, dY, grads, True, ws)
    assert np.array_equal(grads.double().cpu().numpy()[enc:], 2 * g[enc:])
    # nothing to decode: zeros
    tfm.decode_bwd(dims, en, np.full(B, R, np.int32), e.n_feat, Y, to_dev(e.params),
                   to_dev(dlog), dY, grads, False, ws)
    assert not dY.any() and not grads[enc:].any() and bool((grads[:enc] == 7.0).all())


def test_decode_bwd_gives_the_loss_calls_gradients():
    """Fed with the cross entropy's gradient (as a distillation of alpha = 0 forms it), the decoder
    backward gives decode_loss's gradients to float32 rounding."""
    import torch
    from paper_2606_03681_amd import tfm
    w, e = ends_setup("ragged-small-f32", mean=True)
    dims, en = ends_dims(w), ends_struct(e)
    R = w.cfg["R"]
    N = int((R - w.n_train).sum())
    Y = to_dev(np.random.default_rng(6).normal(size=(len(w.n_train), R, w.cfg["C"] + 1,
                                                     w.cfg["E"])).astype(np.float32))
    ws = torch.empty(tfm.ends_workspace_bytes(dims, en), dtype=torch.uint8, device="cuda")
    P, lab = to_dev(e.params), to_dev(e.labels)
    loss, loss2 = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    z = torch.empty((N, e.K), device="cuda")
    dY, dY2, g, g2 = (torch.zeros_like(t) for t in (Y, Y, P, P))
    tfm.decode_loss(dims, en, w.n_train, e.n_feat, e.n_class, lab, Y, P, loss, z, dY, g, False, ws)
    d = tfm.make_distill(N, e.K, 1, e.K, "f32", 1.0, 0.0, 0)
    nc = to_dev(np.repeat(e.n_class, R - w.n_train).astype(np.int32))
    y = to_dev(np.concatenate([e.labels[b][int(n) - e.T:] for b, n in enumerate(w.n_train)]))
    none = torch.full((N, 1), -1, dtype=torch.int32, device="cuda")
    dws = torch.empty(tfm.distill_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    tfm.distill_loss(d, z, none, torch.zeros((N, 1), device="cuda"), None, y, None, nc, loss2, None,
                     z, dws)                                       # in place
    tfm.decode_bwd(dims, en, w.n_train, e.n_feat, Y, P, z, dY2, g2, False, ws)
    assert abs(float(loss[0]) - float(loss2[0])) <= 1e-5 * float(loss[0])
    assert nerr(dY2.cpu().numpy(), dY.cpu().numpy()) <= 1e-5
    assert nerr(g2.cpu().numpy(), g.cpu().numpy()) <= 1e-5


@pytest.mark.parametrize("name,T", [("d16-bf16", 0), ("prenorm-small-bf16", 4)])
def test_draws_from_the_forward_only_path(name, T):
    import torch
    from paper_2606_03681_amd import tfm
    from paper_2606_03681_amd.stack import InferModel, TrainStep
    w, e = ends_setup(name, T=T)
    cols, V = 2, 9
    ids, table = _cats(w, e, cols, V, 5)
    dims, en = ends_dims(w), ends_struct(e)
    x, lab, cat = to_dev(e.x), to_dev(e.labels), to_dev(ids)
    ts = TrainStep(dims, en, w.n_train, e.n_feat, e.n_class, w.params, e.params, e.table,
                   cat_table=table, cat_cols=cols, cat_scale=2.0)
    ts.run(x, lab, cat_ids=cat)
    rows = w.cfg["R"] - w.n_train
    N = int(rows.sum())
    ref = torch.empty((N, e.K), device="cuda")
    tfm.decode_fwd(dims, en, w.n_train, e.n_feat, ts.Y, ts.ends_params, ref, ts.ends_ws)
    im = InferModel(dims, en, w.n_train, e.n_feat, w.params, e.params, e.table, chunk=16,
                    cat_table=table, cat_cols=cols, cat_scale=2.0)
    rng = np.random.default_rng(8)
    u = rng.random(N).astype(np.float32)
    token, lp, logits = im.draw(x, lab, to_dev(u), cat_ids=cat, n_class=e.n_class, temperature=0.7,
                                top_p=0.9)
    assert torch.equal(logits, ref)                    # bit for bit the training forward's
    z = logits.double().cpu().numpy()
    nc = np.repeat(e.n_class, rows)
    f = lambda v: float(np.float32(v))                 # noqa: E731
    for n in range(N):
        t, l = ov.sample_row(z[n, :nc[n]], temperature=f(0.7), top_p=f(0.9), u=float(u[n]))
        assert int(token[n]) == t and abs(float(lp[n]) - l) <= 2.0 ** -24 * abs(l) + 1e-9
    greedy, _, _ = im.draw(x, lab, to_dev(u), cat_ids=cat, temperature=0.0)
    assert torch.equal(greedy.long(), logits.argmax(1))


def test_training_step_without_unlabelled_rows():
    """Every row labelled: no row to learn from, loss and gradients 0."""
    import torch
    from paper_2606_03681_amd.stack import TrainStep
    w, e = ends_setup("d64-f32")
    n_train = np.full_like(w.n_train, w.cfg["R"])
    ids, table = _cats(w, e, 2, 7, 3)
    ts = TrainStep(ends_dims(w), ends_struct(e), n_train, e.n_feat, e.n_class, w.params, e.params,
                   e.table, cat_table=table, cat_cols=2, distill=dict(k=3, alpha=0.5, tail=1))
    teacher = (torch.empty((0, 3), dtype=torch.int32, device="cuda"),
               torch.empty((0, 3), device="cuda"), torch.empty(0, device="cuda"))
    loss = ts.run(to_dev(e.x), to_dev(e.labels), cat_ids=to_dev(ids), teacher=teacher)
    assert float(loss) == 0.0
    for g in [ts.ends_grads, ts.cat_grad] + list(ts.stack.grads):
        assert bool((g == 0).all())
