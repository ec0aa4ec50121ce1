"""The loss at one end of a training step and the orthogonalisation at the other, together with the step: a small encoder trained on masked
tokens through unpack, linear cross entropy, orthogonalisation, pack and Sae.step."""
import pytest
import torch

from paper_2008_05823_b200 import binding as sb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("compressor,orthogonal,amp", [("sign", False, True), ("topk", True, True), ("sign", True, False)])
def test_it_runs(compressor, orthogonal, amp):
    from paper_2008_05823_b200 import train_example as te
    losses, final = te.train_encoder(steps=4, workers=2, compressor=compressor, orthogonal=orthogonal, amp=amp, avg_period=2)
    assert len(losses) == 4 and all(0 < v < 100 for v in losses) and torch.isfinite(final).all()


def test_gradients_are_those_of_the_logits():
    """The model's gradients with the loss from kept logits in torch, in float32: the losses differ by their sums' roundings (64 terms of a
    logit, 1000 classes: 2^-24 (64 / 16 + 1000 / 64 + 64) of at most |z| = 8, and the same again in the softmax), every gradient by as much
    relative to the sum of magnitudes that it is made of; through two layers no factor of it grows beyond 10, so 1e-4 of the norm covers all."""
    from paper_2008_05823_b200 import train_example as te
    torch.manual_seed(1)
    model = te.Encoder(2, 64, 1000, 64, 4).cuda()
    gen = torch.Generator(device="cuda").manual_seed(2)
    tokens, target = te.masked_batch(gen, 1000, 8, 40)
    loss = model(tokens, target)
    loss.backward()
    got = [p.grad.clone() for p in model.parameters()]
    model.zero_grad()
    keep, te.linear_cross_entropy = te.linear_cross_entropy, lambda x, w, t: torch.nn.functional.cross_entropy((x @ w.t()).flatten(0, 1), t.flatten())
    try:
        want = model(tokens, target)
        want.backward()
    finally:
        te.linear_cross_entropy = keep
    assert abs(float(loss.detach()) - float(want.detach())) < 1e-5 * float(want.detach())
    for g, p in zip(got, model.parameters()):
        if float(p.grad.norm()) > 1e-6:              # (a key's bias has none: softmax does not see it)
            assert float((g - p.grad).norm()) < 1e-4 * float(p.grad.norm())


def test_one_worker_is_momentum_descent_on_orthogonal_gradients():
    """K = 1, C = identity, no clipping in effect: three steps of the loop are three steps of SGD with momentum whose layers' gradients are
    the orthogonal factors (by a singular value decomposition and the iteration on the values).  A float32 result is within 5e-5 of
    the exact one; 1e-3 of the update leaves that room through three steps of lr 0.02."""
    from paper_2008_05823_b200 import orthogonal as og
    from paper_2008_05823_b200 import train_example as te
    steps, lr, scale = 3, 0.02, 0.02
    losses, final = te.train_encoder(steps=steps, workers=1, lr=lr, compressor="identity", max_norm=1e9, amp=False, mode=sb.EF, orthogonal=True, scale=scale)
    torch.manual_seed(0)
    model = te.Encoder(2, 64, 1000, 64, 4).cuda()
    start = torch.cat([p.detach().reshape(-1) for p in model.parameters()])
    gen = torch.Generator(device="cuda").manual_seed(1)
    opt = torch.optim.SGD(model.parameters(), lr=lr, momentum=0.9)
    for i in range(steps):
        tokens, target = te.masked_batch(gen, 1000, 16, 48)
        opt.zero_grad()
        loss = model(tokens, target)
        loss.backward()
        for p in model.matrices():
            g = p.grad.double()
            u, s, vt = torch.linalg.svd(g, full_matrices=False)
            s = s / (g.norm() + 1e-7)
            a, b, c = og.COEFFICIENTS
            for _ in range(5):
                s = a * s + b * s ** 3 + c * s ** 5
            p.grad.copy_((u * s) @ vt * scale)
        opt.step()
        assert abs(float(loss.detach()) - losses[i]) < 1e-4 * abs(losses[i])
    want = torch.cat([p.detach().reshape(-1) for p in model.parameters()])
    assert float((final - want).norm()) < 1e-3 * float((want - start).norm())


def test_the_command(monkeypatch, capsys):
    from paper_2008_05823_b200 import train_example as te
    monkeypatch.setattr("sys.argv", ["train_example", "--model", "encoder", "--steps", "2", "--workers", "2", "--layers", "1", "--orthogonal"])
    te.main()
    assert capsys.readouterr().out.count("loss") == 2
    monkeypatch.setattr("sys.argv", ["train_example", "--orthogonal"])
    with pytest.raises(SystemExit):
        te.main()
