"""Tensors that a caller gives the norms for their outputs."""
import pytest
import torch

from paper_2305_16513_amd import binding as B


class Library:
    """Notes the calls, does nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


def test_the_sum_s_tensor_is_passed_on_with_and_without_x(monkeypatch):
    library = Library()
    monkeypatch.setattr(B, "lib", lambda: library)
    monkeypatch.setattr(B, "_calls", None)
    monkeypatch.setattr(B, "_rows", lambda t, *a, **k: t)
    monkeypatch.setattr(B, "_dev", lambda t, name: t)
    monkeypatch.setattr(B, "_stream", lambda s: None)
    r, x, h, w = (torch.zeros(*s) for s in ((2, 8), (2, 8), (2, 8), (8,)))
    for other in (x, None):
        got, _ = B.sws_norm_add(r, w, x=other, h=h)
        assert got is h and library.calls[-1][1][5] == h.data_ptr()
    assert B.sws_norm_add(r, w)[0] is r and library.calls[-1][1][5] is None


@pytest.mark.gpu
def test_a_tensor_for_the_sum_is_filled_without_x_too():
    r, w = torch.randn(5, 72, device="cuda"), torch.randn(72, device="cuda")
    h = torch.full_like(r, 7.0)
    got, n = B.sws_norm_add(r, w, h=h)
    assert got is h and torch.equal(h, r) and torch.equal(n, B.sws_norm_add(r, w)[1])
    with pytest.raises(ValueError):
        B.sws_norm_add(r, w, h=h[:3])
