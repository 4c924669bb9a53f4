"""The users' and the PS's steps around the codec together (pytest -m gpu): the network's gradients against automatic
differentiation in 64 bits, user by user, and a short training run, which has to lower the error and to repeat itself."""
import pytest

pytestmark = pytest.mark.gpu


def test_every_users_gradient():
    import torch
    from paper_2204_08211_amd.examples.local_training import Network
    dev = "cuda:0"
    net = Network(40, 72, 2, 12)
    w = net.start(3, dev)
    gen = torch.Generator(device=dev)
    gen.manual_seed(5)
    w += 0.1 * torch.randn(net.d, generator=gen, device=dev)
    x, dy = torch.randn(3, 50, 40, generator=gen, device=dev), torch.randn(3, 50, 12, generator=gen, device=dev)
    g = torch.zeros(3, net.d + 5, device=dev)
    _, kept = net.forward(w, x)
    net.backward(w, dy, kept, g)
    for u in range(3):
        p = w.double().cpu().requires_grad_()
        part = lambda name: net.part(p, name)  # noqa: E731
        h = x[u].double().cpu()
        norm = lambda h, k: torch.nn.functional.layer_norm(h, (40,), part(f"weight{k}"), part(f"bias{k}"), 1e-5)  # noqa: E731
        for k in range(2):
            h = h + (norm(h, k) @ part(f"up{k}").t()).relu() @ part(f"down{k}").t()
        ((norm(h, "_out") @ part("out").t()) * dy[u].double().cpu()).sum().backward()
        # fp32 passes through five products of up to 72 terms
        assert float((g[u, :net.d].double().cpu() - p.grad).norm() / p.grad.norm()) <= 2.0 ** -17
    assert bool((g[:, net.d:] == 0).all())


def test_training_lowers_the_error_and_repeats_itself():
    from paper_2204_08211_amd.examples.local_training import Network, train
    net = Network(64, 128, 2, 16)
    errors, bits = train(net, users=3, rows=128, iters=40)
    again, _ = train(net, users=3, rows=128, iters=40)
    assert errors[-1] < 0.5 * errors[0] and 1.0 < bits < 9.0
    assert all(abs(a - b) <= 1e-3 * a for a, b in zip(errors, again))
