"""Buffers that the Python calls hand to the library, on the CPU: their bytes lie side by side."""

import numpy as np
import pytest

from paper_2606_03681_amd import tfm


class _OnGpu:
    """A CPU tensor that says it is on the current GPU (nothing is launched for a refused one)."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0

    def data_ptr(self):
        raise AssertionError("a refused buffer's address was taken")


def _buffers(n):
    """n bytes by their number of elements, but not side by side."""
    import torch
    return [torch.zeros(1, dtype=torch.uint8).expand(n), torch.zeros(2 * n, dtype=torch.uint8)[::2],
            torch.zeros((2, n // 2), dtype=torch.uint8).t()]


def test_buffers_that_do_not_lie_side_by_side_are_refused(monkeypatch):
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    c = tfm.make_cache8(2, 32, 64, 10)
    r = tfm.make_cache8_rows(1, 1, 4, "f32", (0, 0, 0), (0, 0, 0))
    a = tfm.make_cache8_query(1, 1, 2, 4, "f32", (0, 0, 32), (0, 0, 32), 1.0)
    x, lens = _OnGpu(torch.zeros((1, 1, 2, 32))), _OnGpu(torch.zeros(1, dtype=torch.int32))
    nb = tfm.cache8_bytes(c)
    good = torch.zeros(nb, dtype=torch.uint8)
    assert tfm._nbytes(good) == nb and tfm._nbytes(good.view(2, -1)) == nb and tfm._nbytes(None) == 0
    monkeypatch.setattr(tfm, "_ptrs", lambda *t: [None] * len(t))   # (what is refused comes first)
    for bad in _buffers(nb):
        assert bad.nbytes == nb
        with pytest.raises(ValueError, match="side by side"):
            tfm.cache8_append(c, r, x, x, None, None, None, _OnGpu(bad), stream=0)
        with pytest.raises(ValueError, match="side by side"):
            tfm.cache8_attend(c, a, x, None, lens, None, _OnGpu(bad), x, None, None, stream=0)
        with pytest.raises(ValueError, match="side by side"):
            tfm.cache8_attend(c, a, x, None, lens, None, _OnGpu(good), x, None, _OnGpu(bad), stream=0)


def test_layer_buffers_that_do_not_lie_side_by_side_are_refused():
    import torch
    d = tfm.make_dims(B=2, R=64, C=8, E=64, heads=4, H=128, dtype="bf16")
    nt, mask = np.full(2, 5, np.int32), np.ones((2, 9), np.uint8)
    x, good = 1 << 20, torch.zeros(64, dtype=torch.uint8)
    for bad in _buffers(1 << 10):
        for bufs in ((bad, good, good), (good, bad, good), (good, good, bad)):
            with pytest.raises(ValueError, match="side by side"):
                tfm.layer_fwd_context8(d, nt, mask, x, x, x, *bufs, stream=0)
        for cache, ws in ((bad, good), (good, bad)):
            with pytest.raises(ValueError, match="side by side"):
                tfm.layer_fwd_query8(d, 32, nt, mask, x, x, cache, x, ws, stream=0)
            with pytest.raises(ValueError, match="side by side"):
                tfm.layer_fwd_query(d, 32, nt, mask, x, x, cache, x, ws, stream=0)
            with pytest.raises(ValueError, match="side by side"):
                tfm.layer_fwd(d, nt, mask, x, x, x, cache, ws, stream=0)
