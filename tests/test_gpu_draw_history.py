"""Histories of draws as a serving loop keeps them: the part of a longer buffer that has been said so
far, or one row for all."""

import numpy as np
import pytest

from oracle import vocab as ov

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K,n", [(1, 7, 3), (5, 10, 1), (40, 64, 9), (6, 10, 0), (0, 10, 4)])
@pytest.mark.parametrize("one", [False, True])
def test_history_of_a_longer_buffer(N, K, n, one):
    import torch
    from paper_2606_03681_amd import stack
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    rng = np.random.default_rng(N + K)
    logits = rng.normal(size=(N, K)).astype(np.float32)
    said = rng.integers(-1, K, (1 if one else N, n + 8)).astype(np.int32)
    buffer = torch.from_numpy(said).cuda()
    history = buffer[:, 2:2 + n]
    history = history.expand(N, n) if one else history
    z = torch.from_numpy(logits.copy()).cuda()
    rep = torch.full((N,), 1.5, device="cuda")
    freq = torch.full((N,), 0.25, device="cuda")
    stack.adjust_classes(z, history=history, repetition=rep, frequency=freq)
    got = z.double().cpu().numpy()
    for r in range(N):
        want, size = ov.adjust_row(logits[r], None, said[0 if one else r, 2:2 + n], 1.5, 0.0, 0.25)
        assert np.all(np.abs(got[r] - want) <= 1.01 * 2.0 ** -24 * size)
    assert np.array_equal(buffer.cpu().numpy(), said)
