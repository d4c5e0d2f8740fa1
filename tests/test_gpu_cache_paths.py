"""Attention over an 8-bit cache (include/tfm_cache.h) where its work is cut: keys in many pieces and
their join, pieces that span more than 64 entries of the page table, workspaces, batches; against the
float64 oracle.

Bounds as derived in test_gpu_cache.py, with h = 2^-11 for weights rounded to half (11 bits, halves to
even: off by half a step, 2^-11 of the power of two below) and 2^-40 of the largest code for values of
blocks far below the largest (half a step of half, 2^-25, of 448 2^7)."""

import numpy as np
import pytest

from oracle import cache as oc

from test_gpu_cache import (U, B, _dev, _ints, _load, _loop, _pool_to_device, _random_pool, _rounded,
                            _step, _table)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    from paper_2606_03681_amd import tfm
    tfm.lib()


def _attend(c, a, qt, pages, lens, n_rows, pool):
    """out (3.25 where nothing is written), lse (9.5), the workspace's bytes."""
    import torch
    from paper_2606_03681_amd import tfm
    nb = tfm.cache8_attend_workspace_bytes(c, a)
    ws = torch.full((nb,), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(qt, 3.25), torch.full((a.B, a.L, a.heads), 9.5, device="cuda")
    tfm.cache8_attend(c, a, qt, _ints(pages), _ints(lens), _ints(n_rows), pool, out, lse, ws)
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), nb


def _check(q, host, page, mp, pages, lens, n_rows, dtype, causal, scale=None, pieces=None):
    """Against the oracle; pieces: whether the keys are in several, by the workspace that they need."""
    from paper_2606_03681_amd import tfm
    Bn, L, H, d = q.shape
    q = _rounded(q, dtype)
    scale = float(np.float32(1 / np.sqrt(d) if scale is None else scale))
    c = tfm.make_cache8(host[0].shape[1], d, page, host[0].shape[0])
    qt = _dev(q, dtype)
    a = tfm.make_cache8_query(Bn, L, H, mp, dtype, qt.stride()[:3], qt.stride()[:3], scale, causal)
    out, lse, nb = _attend(c, a, qt, pages, lens, n_rows, _pool_to_device(*host))
    assert pieces is None or (nb > 0) == pieces
    want, want_lse, mag, sabs, vmax = oc.attend(q, *host, mp, pages, lens, n_rows, scale, causal)
    r = np.full(Bn, L) if n_rows is None else np.clip(n_rows, 0, L)
    live = np.arange(L)[None] < r[:, None]
    assert np.all(out[~live] == 3.25) and np.all(lse[~live] == 9.5)
    n = max(1, min(mp * page, int(np.max(lens))))
    A = (d + 8) * U * sabs
    h = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -23
    e = 4 * A + 16 * U * sabs + 16 * U + h + 2 * (n / 16 + 64) * U
    bound = e[..., None] * mag + n * (2.0 ** -33 + 2.0 ** -40) * vmax[..., None]
    bound = bound + (B if dtype == "bf16" else U) * (np.abs(want) + bound)
    assert np.all(np.abs(out - want)[live] <= bound[live])
    lb = 2 * A + 8 * U * sabs + (n / 16 + 80) * U + 4 * U * np.abs(want_lse)
    some = np.isfinite(want_lse) & live[..., None]
    assert np.all(np.abs(lse[some] - want_lse[some]) <= lb[some])
    assert np.all(lse[np.isinf(want_lse) & live[..., None]] == -np.inf)
    return out, lse


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,page,Bn,L,H,kv,lens,causal", [
    (16, 64, 1, 4, 8, 1, [3000], 0), (32, 16, 2, 6, 6, 2, [2500, 40], 1),
    (64, 64, 1, 32, 2, 2, [2600], 1), (128, 32, 1, 17, 1, 1, [2900], 0),
    (128, 256, 2, 2, 24, 2, [2048, 1025], 1),
])
def test_17_to_32_columns_over_keys_in_pieces(d, page, Bn, L, H, kv, lens, causal, dtype):
    rng = np.random.default_rng(d + L)
    mp = -(-max(lens) // page)
    host = _random_pool(rng, Bn * mp + 1, kv, page, d)
    _check(rng.normal(size=(Bn, L, H, d)), host, page, mp, _table(rng, Bn, mp, Bn * mp + 1), lens,
           None, dtype, causal, pieces=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,page,Bn,L,H,kv,lens,causal", [
    (16, 64, 1, 70, 2, 2, [2300], 1), (16, 16, 2, 33, 2, 1, [2100, 1025], 0),
    (32, 64, 1, 130, 1, 1, [3100], 0), (32, 32, 2, 90, 2, 2, [2200, 0], 1),
    (64, 64, 1, 129, 1, 1, [2500], 1), (64, 16, 1, 70, 2, 1, [2200], 0),
    (128, 32, 1, 40, 1, 1, [2200], 1),
])
def test_many_columns_over_keys_in_pieces(d, page, Bn, L, H, kv, lens, causal, dtype):
    rng = np.random.default_rng(d + L)
    mp = -(-max(lens) // page)
    host = _random_pool(rng, Bn * mp + 1, kv, page, d)
    _check(rng.normal(size=(Bn, L, H, d)), host, page, mp, _table(rng, Bn, mp, Bn * mp + 1), lens,
           np.array([L, L - 3])[:Bn], dtype, causal, pieces=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["rising", "falling", "even"])
@pytest.mark.parametrize("d,n,L", [(128, 45000, 1), (128, 40000, 20), (64, 70000, 1)])
def test_more_pieces_than_a_join_takes_at_a_time(d, n, L, order, dtype):
    """Sums whose reference rises or falls along the pieces: by some 30 from the first to the last."""
    rng = np.random.default_rng(n)
    page = 256
    mp = -(-n // page)
    host = _random_pool(rng, mp, 1, page, d, (116, 117))
    if order != "even":
        size = np.linspace(0.02, 1, mp * page)[::1 if order == "rising" else -1]
        x = np.broadcast_to(size[:, None], (mp * page, d)).reshape(mp, 1, page, d)
        host[0][:] = oc.encode(x * 440)
    q = np.abs(rng.normal(size=(1, L, 1, d)))
    _check(q, host, page, mp, _table(rng, 1, mp, mp), [n], None, dtype, 0,
           scale=0.2 if order == "even" else 30 / (440 * 2.0 ** -11 * d * 0.8), pieces=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,page,Bn,L,H,kv,n,causal", [
    (32, 16, 256, 1, 8, 4, 2600, 0),        # two pieces of 96 entries, four waves in turn
    (64, 16, 512, 3, 4, 4, 4200, 1),        # one of 263
    (32, 16, 128, 40, 4, 4, 2600, 1), (128, 32, 512, 40, 4, 4, 5000, 0),
    (64, 32, 512, 34, 4, 4, 5000, 1), (32, 64, 512, 1, 4, 4, 9000, 0),
    (128, 64, 512, 70, 4, 4, 5000, 1),      # bfloat16: tiles that a workgroup reads together
])
def test_pieces_of_more_than_64_pages(d, page, Bn, L, H, kv, n, causal, dtype):
    """Enough sequences for long pieces; three of them have keys, on pages in any order, some absent."""
    rng = np.random.default_rng(d + page + L)
    mp, n_pages = -(-n // page), 400
    host = _random_pool(rng, n_pages, kv, page, d)
    pages = rng.integers(0, n_pages, (Bn, mp)).astype(np.int32)
    pages[rng.random(pages.shape) < 0.05] = -1
    lens, n_rows = np.zeros(Bn, int), np.zeros(Bn, int)
    for b, m in ((0, n), (Bn // 2, n - 1000), (Bn - 1, 1030)):
        lens[b], n_rows[b] = m, min(L, 5)
    n_rows[0] = L if L > 5 and d < 128 else n_rows[0]
    _check(rng.normal(size=(Bn, L, H, d)), host, page, mp, pages, lens, n_rows, dtype, causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_row_in_batches_of_many_sizes(dtype):
    """The same sequence alone, with others, and among so many that its keys are not split."""
    rng = np.random.default_rng(7)
    mp, page, n = 20, 64, 1250
    host = _random_pool(rng, 60, 2, page, 64)
    own, q0 = rng.permutation(60)[:mp], rng.normal(size=(3, 4, 64))
    for Bn, at in ((1, 0), (3, 1), (64, 63), (1100, 500)):
        pages = rng.integers(0, 60, (Bn, mp)).astype(np.int32)
        q, lens = rng.normal(size=(Bn, 3, 4, 64)), np.zeros(Bn, int)
        pages[at], q[at], lens[at] = own, q0, n
        lens[:2] = np.maximum(lens[:2], 5)
        _check(q, host, page, mp, pages, lens, None if Bn < 4 else (lens > 0) * 3, dtype, 1,
               pieces=Bn < 1100)


def test_calls_on_two_streams_with_workspaces_of_their_own():
    import torch
    n, shape = 10, (16, 4, 128, 64, 40, 5)
    H, kv, d, page, mp, Bn = shape

    def loop(seed):
        s = _loop(n, *shape, seed)
        rng = np.random.default_rng(seed)
        s["pool"].copy_(_pool_to_device(*_random_pool(rng, Bn * mp, kv, page, d)))
        s["lens"].copy_(_ints(rng.integers(1500, 2500, Bn)))
        assert s["ws"].numel() > 0
        return s

    want = []
    for seed in (3, 4):
        s = loop(seed)
        outs = []
        for i in range(n):
            _load(s, i)
            _step(s)
            outs.append(s["out"].clone())
        want.append((outs, s["pool"].clone()))
    loops = [loop(seed) for seed in (3, 4)]
    got = [[], []]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(n):
        for s, st, o in zip(loops, streams, got):
            with torch.cuda.stream(st):
                _load(s, i)
                _step(s)
                o.append(s["out"].clone())
    torch.cuda.synchronize()
    for s, o, (outs, pool) in zip(loops, got, want):
        assert all(torch.equal(x, y) for x, y in zip(o, outs)) and torch.equal(s["pool"], pool)
