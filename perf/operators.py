"""The operators over discrete values at the two ends of the stack, as calls to time and compare.

  embed_fwd   rows of an embedding table, scaled, at given ids (include/tfm_vocab.h)
  embed_bwd   the table's gradient: the rows of every id summed
  distill     a teacher's top logits against the student's logits: loss and gradient
  sample      one draw per row under temperature, top-k, top-p and min-p from given uniforms

run() computes them from elementary torch operations, or through the package's entry points where
`own` is true; exact() holds their definitions in 64 bits.  Notation: an id or a class outside the
range is absent; a row without an admissible class has no loss, no gradient and no token.
"""

import math

import numpy as np
import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------

def _embed(op, n0, n1, n2, cells, V, E, table, rows, skew, name=None):
    """ids [n0][n1][n2]; cells > 0: the rows are the first n2 cells of stack rows of that many
    cells, 0: rows side by side.  table, rows: types.  skew: the ids' density falls as rank grows
    (0: even)."""
    c = dict(op=op, n0=n0, n1=n1, n2=n2, cells=cells, V=V, E=E, table=table, rows=rows, skew=skew)
    return dict(name=name, **c) if name else c


def _distill(N, V, k, dtype, tail, temperature, alpha, classes=0, weights=0, pad=0, name=None):
    """classes: rows have 2 .. V classes; weights: a tenth of the rows weighs nothing; pad:
    elements between the rows."""
    c = dict(op="distill", N=N, V=V, k=k, dtype=dtype, tail=tail, temperature=temperature,
             alpha=alpha, classes=classes, weights=weights, pad=pad)
    return dict(name=name, **c) if name else c


def _sample(N, V, dtype, mode, classes=0, pad=0, name=None):
    """mode: "plain" (temperature alone), "k", "p", "kp", "min", or "mixed" (each row its own)."""
    c = dict(op="sample", N=N, V=V, dtype=dtype, mode=mode, classes=classes, pad=pad)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # serving: the tokens of one step of sixteen sequences
        _embed("embed_fwd", 1, 1, 16, 0, 32000, 2048, "bf16", "bf16", 1.0, "embed-step"),
        # twenty categorical columns of the evaluation batch, written into the stack input
        _embed("embed_fwd", 16, 1024, 20, 101, 997, 192, "f32", "bf16", 0.5, "embed-table"),
        # and the gradient of their table: few categories, each in thousands of cells
        _embed("embed_bwd", 16, 1024, 20, 101, 997, 192, "f32", "bf16", 0.5, "embed-table-grad"),
        # a text batch against a large vocabulary: most ids rare, a few in every sentence
        _embed("embed_bwd", 1, 1, 40001, 0, 50021, 1024, "f32", "bf16", 1.0, "embed-text-grad"),
        # the unlabelled rows of the evaluation batch: ten classes, a teacher's five best
        _distill(4096, 10, 5, "f32", 0, 2.0, 0.7, classes=1, name="distill-classes"),
        # a regression head of 5,000 buckets, everything from the teacher
        _distill(8192, 5000, 32, "f32", 1, 1.0, 1.0, name="distill-buckets"),
        # text: a large odd vocabulary, labels mixed in, padding rows of weight 0
        _distill(4096, 50021, 64, "bf16", 1, 1.5, 0.5, weights=1, name="distill-text"),
        # few rows of a long vocabulary: latency and too few rows to fill the chip
        _distill(7, 131072, 256, "bf16", 1, 2.0, 1.0, name="distill-few"),
        # serving one sequence
        _sample(1, 32000, "f32", "kp", name="sample-one"),
        # class draws for the unlabelled rows of the evaluation batch
        _sample(4096, 10, "f32", "plain", classes=1, name="sample-classes"),
        # a serving batch, each request with settings of its own
        _sample(64, 131072, "bf16", "mixed", name="sample-batch"),
        # draws from a regression head's buckets
        _sample(8192, 5000, "f32", "p", name="sample-buckets"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: 1 .. 65,536 rows, 2 .. 131,072 classes, widths 32 .. 4,096."""
    top = {}
    for c in listed():
        top[c["op"]] = max(top.get(c["op"], 0), _cost(c))
    op = rng.choice(["embed_fwd", "embed_bwd", "distill", "sample"])
    while True:
        if op in ("embed_fwd", "embed_bwd"):
            table, rows = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
            if rng.random() < 0.5:
                n2 = _log_int(rng, 1, 40)
                c = _embed(op, _log_int(rng, 1, 32), _log_int(rng, 1, 2000), n2,
                           n2 + rng.randint(1, 20), _log_int(rng, 2, 5000),
                           rng.choice([64, 96, 192, 256]), table, rows, rng.choice([0.0, 0.5, 1.0]))
            else:
                c = _embed(op, 1, 1, _log_int(rng, 1, 65536), 0, _log_int(rng, 100, 131072),
                           rng.choice([_log_int(rng, 32, 4096), 8 * _log_int(rng, 4, 512)]), table,
                           rows, rng.choice([0.0, 0.5, 1.0]))
            if c["V"] * c["E"] > 60_000_000:
                continue
        else:
            small = rng.random() < 0.4
            N = _log_int(rng, 1, 65536)
            V = _log_int(rng, 2, 64) if small else _log_int(rng, 65, 131072)
            dtype = rng.choice(["f32", "bf16"])
            classes, pad = int(small and rng.random() < 0.7), rng.choice([0, 0, 0, 1, 24])
            if op == "distill":
                alpha = rng.choice([1.0, 0.5, 0.9])
                c = _distill(N, V, _log_int(rng, 1, min(256, V)), dtype, rng.randint(0, 1),
                             rng.choice([1.0, 2.0, 0.7, 4.0]), alpha, classes, rng.randint(0, 1),
                             pad)
            else:
                c = _sample(N, V, dtype, rng.choice(["plain", "k", "p", "kp", "min", "mixed"]),
                            classes, pad)
        if _cost(c) <= top[op]:
            return c


def _cost(c):
    if c["op"].startswith("embed"):
        return c["n0"] * c["n1"] * c["n2"] * c["E"] + c["V"] * c["E"] * (c["op"] == "embed_bwd")
    return c["N"] * c["V"]


def work(case):
    """Each input read once and each output written once; flops count the exponentials as one."""
    if case["op"].startswith("embed"):
        n, E, V = case["n0"] * case["n1"] * case["n2"], case["E"], case["V"]
        rows = n * E * SIZE[case["rows"]]
        if case["op"] == "embed_fwd":
            return {"bytes": 4 * n + min(n, V) * E * SIZE[case["table"]] + rows, "flops": n * E}
        return {"bytes": 4 * n + rows + 4 * V * E, "flops": n * E + V * E}
    el = case["N"] * case["V"]
    if case["op"] == "distill":
        return {"bytes": 2 * el * SIZE[case["dtype"]] + case["N"] * (8 * case["k"] + 16),
                "flops": el * (8 if case["alpha"] == 1.0 else 12)}
    return {"bytes": el * SIZE[case["dtype"]] + 28 * case["N"], "flops": 6 * el}


# ---------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed * 7919 + 17)
    if case["op"].startswith("embed"):
        return _prepare_embed(case, g)
    return (_prepare_distill if case["op"] == "distill" else _prepare_sample)(case, g)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEVICE)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _prepare_embed(case, g):
    n0, n1, n2, V, E = (case[k] for k in ("n0", "n1", "n2", "V", "E"))
    # id density ~ rank^-skew by inverting its integral; a fiftieth of the ids is absent
    u = _rand(g, n0, n1, n2).double()
    a = case["skew"]
    x = V ** u if a == 1.0 else (u * (V ** (1 - a) - 1) + 1) ** (1 / (1 - a))
    ids = (x.long() - 1).clamp_(0, V - 1)
    ids = torch.randperm(V, generator=g, device=DEVICE)[ids]
    ids = torch.where(_rand(g, n0, n1, n2) < 0.02, -1, ids).to(torch.int32)
    cells = case["cells"] or n2
    rows = torch.zeros((n0, n1, cells, E), dtype=TORCH[case["rows"]], device=DEVICE)
    s = dict(case=case, ids=ids, rows=rows, scale=math.sqrt(E))
    if case["op"] == "embed_fwd":
        s["table"] = (0.02 * _randn(g, V, E)).to(TORCH[case["table"]])
    else:
        rows.copy_(1e-3 * _randn(g, n0, n1, cells, E))
        s["dtable"] = torch.empty((V, E), dtype=torch.float32, device=DEVICE)
    return s


def _spiked(g, N, V):
    """Logits of a trained head: a broad floor and a few classes that stand out."""
    z = 2.0 * _randn(g, N, V)
    m = max(1, min(40, V // 4))
    at = torch.randint(0, V, (N, m), generator=g, device=DEVICE)
    z.scatter_add_(1, at, 4.0 + 3.0 * _randn(g, N, m))
    return z


def _in_rows(z, dtype, pad):
    """z as rows with `pad` elements between them."""
    N, V = z.shape
    buf = torch.zeros((N, V + pad), dtype=TORCH[dtype], device=DEVICE)
    buf[:, :V] = z
    return buf[:, :V]


def _classes(case, g):
    if not case["classes"]:
        return None
    return torch.randint(min(2, case["V"]), case["V"] + 1, (case["N"],), generator=g,
                         device=DEVICE).to(torch.int32)


def _prepare_distill(case, g):
    N, V, k, tau = case["N"], case["V"], case["k"], case["temperature"]
    nc = _classes(case, g)
    t = _spiked(g, N, V)
    logits = _in_rows(0.8 * t + 0.7 * _randn(g, N, V), case["dtype"], case["pad"])
    if nc is not None:
        t = torch.where(torch.arange(V, device=DEVICE) < nc[:, None], t, -math.inf)
    val, idx = torch.topk(t, k, dim=1)
    idx = torch.where(val > -math.inf, idx, -1).to(torch.int32)
    lse = torch.logsumexp(t / tau, 1)
    labels = idx[:, 0].clone()
    labels[_rand(g, N) < 0.1] = -1
    w = None
    if case["weights"]:
        w = (0.5 + _rand(g, N)) * (_rand(g, N) >= 0.1)
    return dict(case=case, logits=logits, n_class=nc, top_idx=idx.contiguous(),
                top_logit=val.contiguous(), top_lse=lse.contiguous(),
                labels=labels if case["alpha"] < 1 else None, weights=w,
                loss=torch.empty(4, dtype=torch.float32, device=DEVICE),
                row_loss=torch.empty(N, dtype=torch.float32, device=DEVICE),
                dlogits=torch.zeros_like(logits.as_strided((N, V + case["pad"]),
                                                           (V + case["pad"], 1)))[:, :V])


def _prepare_sample(case, g):
    N, V, mode = case["N"], case["V"], case["mode"]
    s = dict(case=case, logits=_in_rows(_spiked(g, N, V), case["dtype"], case["pad"]),
             n_class=_classes(case, g), u=_rand(g, N),
             temperature=0.6 + 0.8 * _rand(g, N), top_k=None, top_p=None, min_p=None,
             token=torch.empty(N, dtype=torch.int32, device=DEVICE),
             logprob=torch.empty(N, dtype=torch.float32, device=DEVICE))
    if mode in ("k", "kp", "mixed"):
        s["top_k"] = torch.randint(1, 100, (N,), generator=g, device=DEVICE).to(torch.int32)
    if mode in ("p", "kp", "mixed"):
        s["top_p"] = 0.5 + 0.48 * _rand(g, N)
    if mode in ("min", "mixed"):
        s["min_p"] = 0.1 * _rand(g, N)
    if mode == "mixed":  # some rows without one filter or another, some greedy
        s["temperature"] = torch.where(_rand(g, N) < 0.1, 0.0, s["temperature"])
        s["top_k"] = torch.where(_rand(g, N) < 0.5, 0, s["top_k"])
        s["top_p"] = torch.where(_rand(g, N) < 0.3, 1.0, s["top_p"])
        s["min_p"] = torch.where(_rand(g, N) < 0.5, 0.0, s["min_p"])
    return s


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if op == "embed_fwd":
        return _own_embed_fwd(state) if own else _plain_embed_fwd(state)
    if op == "embed_bwd":
        return _own_embed_bwd(state) if own else _plain_embed_bwd(state)
    if op == "distill":
        return _own_distill(state) if own else _plain_distill(state)
    return _own_sample(state) if own else _plain_sample(state)


def _workspace(state, nbytes):
    if "workspace" not in state:
        state["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device=DEVICE)
    return state["workspace"]


def _own_embed_shape(state):
    from paper_2606_03681_amd import tfm
    c, rows = state["case"], state["rows"]
    return tfm.make_embed((c["n0"], c["n1"], c["n2"]), rows.stride()[:3], c["E"], c["V"],
                          c["rows"], c["table"], state["scale"])


def _own_embed_fwd(state):
    from paper_2606_03681_amd import tfm
    tfm.embed_fwd(_own_embed_shape(state), state["ids"], state["table"], state["rows"])
    return state["rows"][:, :, :state["case"]["n2"]]


def _own_embed_bwd(state):
    from paper_2606_03681_amd import tfm
    e = _own_embed_shape(state)
    tfm.embed_bwd(e, state["ids"], state["rows"], state["dtable"], False,
                  _workspace(state, tfm.embed_workspace_bytes(e)))
    return state["dtable"]


def _own_distill(state):
    from paper_2606_03681_amd import tfm
    c = state["case"]
    d = tfm.make_distill(c["N"], c["V"], c["k"], c["V"] + c["pad"], c["dtype"], c["temperature"],
                         c["alpha"], c["tail"])
    tfm.distill_loss(d, state["logits"], state["top_idx"], state["top_logit"],
                     state["top_lse"] if c["tail"] else None, state["labels"], state["weights"],
                     state["n_class"], state["loss"], state["row_loss"], state["dlogits"],
                     _workspace(state, tfm.distill_workspace_bytes(d)))
    return {"loss": state["loss"][:1], "row_loss": state["row_loss"],
            "dlogits": state["dlogits"]}


def _own_sample(state):
    from paper_2606_03681_amd import tfm
    c = state["case"]
    tfm.sample(tfm.make_sampling(c["N"], c["V"], c["V"] + c["pad"], c["dtype"]), state["logits"],
               state["n_class"], state["temperature"], state["top_k"], state["top_p"],
               state["min_p"], state["u"], state["token"], state["logprob"])
    return {"token": state["token"], "logprob": state["logprob"]}


def _plain_embed_fwd(state):
    ids = state["ids"].long()
    here = (ids >= 0) & (ids < state["case"]["V"])
    rows = state["table"][ids.clamp(0, state["case"]["V"] - 1)].float() * state["scale"]
    return torch.where(here[..., None], rows, 0.0).to(TORCH[state["case"]["rows"]])


def _plain_embed_bwd(state):
    c = state["case"]
    V = c["V"]
    ids = state["ids"].long().reshape(-1)
    ids = torch.where((ids >= 0) & (ids < V), ids, V)
    d = state["rows"][:, :, :c["n2"]].reshape(-1, c["E"]).float()
    sums = torch.zeros((V + 1, c["E"]), dtype=torch.float32, device=d.device).index_add_(0, ids, d)
    return sums[:V] * state["scale"]


def _plain_distill(state):
    """The rows' scalars in 64 bits: the loss is a small difference of large logarithms where the
    student is near the teacher."""
    c = state["case"]
    V, tau, alpha = c["V"], float(np.float32(c["temperature"])), float(np.float32(c["alpha"]))
    s = state["logits"].float()
    if state["n_class"] is not None:
        s = torch.where(torch.arange(V, device=s.device) < state["n_class"][:, None], s, -math.inf)
    last = s.shape[1] if state["n_class"] is None else state["n_class"][:, None]
    idx = state["top_idx"].long()
    here = (idx >= 0) & (idx < last)
    at = idx.clamp(0, V - 1)
    t = torch.where(here, state["top_logit"], -math.inf).double() / tau
    if c["tail"]:
        p = torch.exp(t - state["top_lse"].double()[:, None])
    else:
        p = torch.exp(t - t.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        p = torch.where(here, p, 0.0)
    inside = torch.zeros_like(s, dtype=torch.int32).scatter_add_(1, at, here.int()) > 0
    sj = torch.where(here, s.gather(1, at), -math.inf).double()
    m = s.amax(1, keepdim=True)
    # one sum over the classes outside the top set, one over those in it
    mt = torch.where(inside, -math.inf, s).amax(1, keepdim=True)
    some = mt > -math.inf
    mt = torch.where(some, mt, 0.0)
    et = torch.where(inside, 0.0, torch.exp((s - mt) / tau))
    st = et.sum(1, keepdim=True)
    far = torch.exp((mt - m).double() / tau)
    total = far * st.double() + torch.exp((sj - m) / tau).sum(1, keepdim=True)
    lq = (sj - m) / tau - torch.log(total)
    D = torch.where(p > 0, p * (torch.log(p) - lq), 0.0).sum(1)
    P = p.sum(1, keepdim=True)
    rest = torch.zeros_like(P)
    if c["tail"]:
        rest = torch.where(some, (1 - P).clamp(min=0), 0.0)
        lqt = (mt - m).double() / tau + torch.log(st.double()) - torch.log(total)
        D = D + torch.where(rest > 0, rest * (torch.log(rest) - lqt), 0.0)[:, 0]
    q = torch.exp((s - m) / tau) / total.float()
    grad = q * (P + rest).float() - torch.where(some, rest.float() * et / st, 0.0)
    grad = alpha * tau * grad.scatter_add(1, at, -torch.where(here, p, 0.0).float())
    L = alpha * tau * tau * D
    if state["labels"] is not None:
        y = state["labels"].long()[:, None]
        known = ((y >= 0) & (y < last)).float()
        y = y.clamp(0, V - 1)
        e1 = torch.exp(s - m)
        z1 = e1.sum(1, keepdim=True)
        nll = torch.log(z1.double()) - (s.gather(1, y) - m).double()
        L = L + (1 - alpha) * (known * nll)[:, 0]
        grad = grad + (1 - alpha) * known * (e1 / z1).scatter_add(1, y, -torch.ones_like(known))
    w = state["weights"]
    w = torch.ones(c["N"], device=s.device).double() if w is None else w.double()
    L = torch.where(w != 0, L, 0.0)
    share = w / torch.where(w.sum() != 0, w.sum(), 1.0)
    loss = (share * L.double()).sum()
    grad = torch.where(w[:, None] != 0, grad * share.float()[:, None], 0)
    return {"loss": loss.float().reshape(1), "row_loss": L.float(),
            "dlogits": grad.to(TORCH[c["dtype"]])}


def _plain_sample(state):
    """In 64 bits throughout: a border between two classes decides which one is drawn."""
    c = state["case"]
    N, V = c["N"], c["V"]
    s = state["logits"].float()
    place = torch.arange(V, device=s.device)
    if state["n_class"] is not None:
        s = torch.where(place < state["n_class"][:, None], s, -math.inf)
    order_s, order = torch.sort(s, dim=1, descending=True, stable=True)
    tau = state["temperature"].double()[:, None]
    greedy = tau <= 0
    top = order_s[:, :1].double()
    x = (order_s.double() - top) / torch.where(greedy, 1.0, tau)
    w = torch.exp(x)
    keep = torch.where(greedy, place == 0, order_s > -math.inf)
    if state["top_k"] is not None:
        k = state["top_k"].long()[:, None]
        keep &= (place < k) | (k <= 0)
    if state["top_p"] is not None:
        wk = torch.where(keep, w, 0.0)
        before = torch.cumsum(wk, 1) - wk
        p = state["top_p"].double()[:, None]
        keep &= (before < p * wk.sum(1, keepdim=True)) | (p >= 1) | (place == 0)
    if state["min_p"] is not None:
        m = state["min_p"].double()[:, None]
        keep &= (x >= torch.log(m)) | (m <= 0) | (place == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))
    mass = torch.cumsum(w, 1)
    target = state["u"].double()[:, None] * mass[:, -1:]
    token = (mass <= target).sum(1).clamp(max=V - 1)
    xi = torch.zeros_like(w).scatter_(1, order, x).gather(1, token[:, None])
    return {"token": token.to(torch.int32),
            "logprob": (xi - torch.log(mass[:, -1:]))[:, 0].float()}


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------

def exact(case, seed):
    if _cost(case) > 220_000_000 or (case["op"] == "sample" and case["N"] > 20000):
        return None
    s = prepare(case, seed)
    if case["op"].startswith("embed"):
        return _exact_embed(case, s)
    return (_exact_distill if case["op"] == "distill" else _exact_sample)(case, s)


def _exact_embed(case, s):
    """As a product with the ids' one-hot rows would give it, in order of the ids."""
    V, E = case["V"], case["E"]
    ids = s["ids"].reshape(-1).cpu().numpy().astype(np.int64)
    scale = float(np.float32(s["scale"]))
    known = np.flatnonzero((ids >= 0) & (ids < V))
    if case["op"] == "embed_fwd":
        out = np.zeros((len(ids), E))
        out[known] = s["table"].double().cpu().numpy()[ids[known]] * scale
        return out.reshape(case["n0"], case["n1"], case["n2"], E)
    d = s["rows"][:, :, :case["n2"]].double().cpu().numpy().reshape(len(ids), E)
    out = np.zeros((V, E))
    if len(known):
        by = known[np.argsort(ids[known], kind="stable")]
        heads = np.flatnonzero(np.diff(ids[by], prepend=-1))
        out[ids[by][heads]] = np.add.reduceat(d[by], heads, axis=0) * scale
    return out


def _exact_distill(case, s):
    """Row block by row block from log-sum-exps; gradients as differences of distributions."""
    N, V, tau, alpha = case["N"], case["V"], case["temperature"], case["alpha"]
    tau, alpha = float(np.float32(tau)), float(np.float32(alpha))
    w = torch.ones(N, device=DEVICE) if s["weights"] is None else s["weights"]
    w = w.double() / (w.double().sum() if w.any() else 1.0)
    rows, grads = [], []
    for a in range(0, N, 1024):
        b = min(N, a + 1024)
        z = s["logits"][a:b].double()
        nc = torch.full((b - a,), V, device=DEVICE) if s["n_class"] is None else \
            s["n_class"][a:b].long()
        z = z.masked_fill(torch.arange(V, device=DEVICE)[None] >= nc[:, None], -math.inf)
        idx = s["top_idx"][a:b].long()
        ok = (idx >= 0) & (idx < nc[:, None])
        idx = idx.clamp(0, V - 1)
        lt = s["top_logit"][a:b].double().masked_fill(~ok, -math.inf) / tau
        norm = s["top_lse"][a:b].double() if case["tail"] else torch.logsumexp(lt, 1)
        lt = lt - norm[:, None]
        lq = torch.log_softmax(z / tau, 1)
        # the teacher's distribution over the classes, its rest spread as the student spreads it
        p = torch.zeros_like(z).scatter_add_(1, idx, torch.exp(lt))
        top = torch.where(ok, torch.exp(lt) * (lt - lq.gather(1, idx)), 0.0).sum(1)
        if case["tail"]:
            out = lq.scatter_add(1, idx, torch.where(ok, -math.inf, 0.0).double())
            lqt = torch.logsumexp(out, 1)
            rest = (1 - torch.exp(lt).sum(1)).clamp(min=0)
            rest = torch.where(lqt == -math.inf, 0.0, rest)
            top = top + torch.where(rest > 0, rest * (torch.log(rest) - lqt), 0.0)
            p = p + torch.where(rest[:, None] > 0, torch.exp(out - lqt[:, None]), 0) * \
                rest[:, None]
        row = alpha * tau * tau * top
        grad = alpha * tau * (torch.exp(lq) * p.sum(1, keepdim=True) - p)
        if s["labels"] is not None:
            y = s["labels"][a:b].long()
            ok = (y >= 0) & (y < nc)
            l1 = torch.log_softmax(z, 1)
            hot = torch.nn.functional.one_hot(y.clamp(0, V - 1), V)
            row = row - (1 - alpha) * ok * l1.gather(1, y.clamp(0, V - 1)[:, None])[:, 0]
            grad = grad + (1 - alpha) * ok[:, None] * (torch.exp(l1) - hot)
        wn = w[a:b]
        rows.append(torch.where(wn != 0, row, 0.0))
        grads.append(torch.where(wn[:, None] != 0, grad * wn[:, None], 0.0))
    rows = torch.cat(rows)
    return {"loss": (w * rows).sum().reshape(1), "row_loss": rows,
            "dlogits": torch.cat(grads)}


def _exact_sample(case, s):
    """Row by row: classes ranked, kept from the front while every rule allows, then walked in
    order of their numbers."""
    z = s["logits"].double().cpu().numpy()
    host = {k: None if s[k] is None else s[k].double().cpu().numpy()
            for k in ("n_class", "temperature", "top_k", "top_p", "min_p", "u")}
    tokens, logs = np.zeros(case["N"], np.int32), np.zeros(case["N"])
    for n in range(case["N"]):
        row = z[n] if host["n_class"] is None else z[n, :int(host["n_class"][n])]
        rank = np.argsort(-row, kind="stable")
        if host["temperature"][n] <= 0:
            tokens[n] = rank[0]
            continue
        x = (row[rank] - row[rank[0]]) / host["temperature"][n]
        w = np.exp(x)
        count = len(row)
        if host["top_k"] is not None and host["top_k"][n] > 0:
            count = min(count, int(host["top_k"][n]))
        if host["top_p"] is not None and host["top_p"][n] < 1:
            mass = np.concatenate([[0.0], np.cumsum(w[:count])])
            count = max(1, int(np.searchsorted(mass[:-1], host["top_p"][n] * mass[-1])))
        if host["min_p"] is not None and host["min_p"][n] > 0:
            count = min(count, max(1, int((x >= math.log(host["min_p"][n])).sum())))
        kept = np.sort(rank[:count])
        mass = np.cumsum(np.exp((row[kept] - row[rank[0]]) / host["temperature"][n]))
        at = min(int(np.searchsorted(mass, host["u"][n] * mass[-1], side="right")), count - 1)
        tokens[n] = kept[at]
        logs[n] = (row[kept[at]] - row[rank[0]]) / host["temperature"][n] - math.log(mass[-1])
    return {"token": tokens, "logprob": logs}
