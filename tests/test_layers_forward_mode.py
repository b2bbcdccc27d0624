"""The layers as autograd functions have no rule for tangents: forward-mode differentiation is refused, with gradients on and off, and
never loses a tangent without a word."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad


def calls(layers, x):
    weight, gate, down = torch.ones(2, 4).to(x), torch.ones(2, 5, 4).to(x), torch.ones(2, 4, 5).to(x)
    return {
        "x of layer_norm": lambda t: layers.layer_norm(t, weight), "weight of layer_norm": lambda t: layers.layer_norm(x, t[:, 0]),
        "x of gated_ffn": lambda t: layers.gated_ffn(t, gate, gate, down), "x of dropout": lambda t: layers.dropout(t, 0.5, 1),
        "residual of dropout": lambda t: layers.dropout(x, 0.5, 1, residual=t)}


def check_refused(layers, x):
    for name, call in calls(layers, x).items():
        for mode in (torch.enable_grad, torch.no_grad):
            with forward_ad.dual_level(), mode():
                with pytest.raises(NotImplementedError):
                    call(forward_ad.make_dual(x, torch.ones_like(x)))
                    pytest.fail(name)
            with mode():
                assert not call(x).requires_grad and call(x.clone().requires_grad_()).requires_grad == (mode is torch.enable_grad), name


def test_tangents_are_refused(monkeypatch):
    """Plain torch in the place of the kernels: what is tested is what lies around them."""
    from paper_2306_06528_amd import layers
    monkeypatch.setattr(layers, "layer_norm_forward", lambda x, weight, bias, eps: (x * weight[:, None], x[..., 0], x[..., 0]))
    monkeypatch.setattr(layers, "gated_ffn_forward", lambda x, gate, up, down, activation, save=False: (x * 2, x * 3 if save else None))
    monkeypatch.setattr(layers, "dropout_forward", lambda x, p, seed, call, residual, counter: x * 2)
    check_refused(layers, torch.ones(2, 3, 4))


@pytest.mark.parametrize("enabled", [True, False])
def test_what_is_kept(monkeypatch, enabled):
    """g, u and h are kept, and the counter is copied, only where a backward pass can follow."""
    from paper_2306_06528_amd import layers
    saves = []
    monkeypatch.setattr(layers, "gated_ffn_forward", lambda x, gate, up, down, activation, save=False: (saves.append(save) or x * 2, x * 3 if save else None))
    monkeypatch.setattr(layers, "dropout_forward", lambda x, p, seed, call, residual, counter: x * 2)

    class Counter:
        copies = 0

        def clone(self):
            self.copies += 1
            return self

    x, p, counter = torch.ones(2, 3, 4, requires_grad=True), torch.ones(1), Counter()
    with torch.set_grad_enabled(enabled):
        layers.gated_ffn(x, p, p, p)
        layers.gated_ffn(x.detach(), p, p, p)
        layers.dropout(x, 0.5, 1, counter=counter)
    assert saves == [enabled, False] and counter.copies == enabled


@pytest.mark.gpu
def test_tangents_are_refused_on_the_gpu():
    from paper_2306_06528_amd import layers
    check_refused(layers, torch.ones(2, 3, 4, device="cuda"))


def test_tangents_of_function_transforms_are_refused(monkeypatch):
    from paper_2306_06528_amd import layers
    monkeypatch.setattr(layers, "dropout_forward", lambda x, p, seed, call, residual, counter: x * 2)

    def quiet(x):
        with torch.no_grad():
            return layers.dropout(x, 0.5, 1)

    x = torch.ones(2, 3, 4)
    assert torch.equal(quiet(x), 2 * x)
    for f in (quiet, lambda t: layers.dropout(t, 0.5, 1)):
        with pytest.raises((NotImplementedError, RuntimeError)):
            torch.func.jvp(f, (x,), (x,))
