"""What the attention half's autograd functions do not differentiate is refused, never left out without a word.  Plain torch in the place of the kernels."""
import pytest
import torch


def test_frequencies_are_no_parameters(monkeypatch):
    from paper_2306_06528_amd import attention
    monkeypatch.setattr(attention, "qk_norm_rotary_forward", lambda q, k, *rest: (q * 2, k * 2))
    q, k = torch.ones(1, 1, 2, 2, 4, requires_grad=True), torch.ones(1, 1, 2, 1, 4)
    f, positions = torch.ones(2, dtype=torch.float64, requires_grad=True), torch.arange(2)
    with pytest.raises(ValueError, match="frequencies"):
        attention.qk_norm_rotary(q, k, None, None, f, positions)
    with pytest.raises(ValueError, match="frequencies"):
        attention.qk_norm_rotary(q.detach(), k, frequencies=f * 2, positions=positions)
    assert attention.qk_norm_rotary(q, k, None, None, f.detach(), positions)[0].requires_grad
    assert attention.qk_norm_rotary(q, k)[0].requires_grad
    with torch.no_grad():
        assert not attention.qk_norm_rotary(q, k, None, None, f, positions)[0].requires_grad
