"""The operators together with the step they stand beside: a small ResNet with group norm trained through unpack, group norm,
pack and Sae.step."""
import pytest
import torch

from paper_2008_05823_b200 import binding as sb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("compressor,avg_period", [("sign", 0), ("sign", 1), ("topk", 5)])
def test_the_loss_falls(compressor, avg_period):
    from paper_2008_05823_b200 import train_example
    losses, final = train_example.train(steps=25, workers=2, blocks=1, classes=4, batch_size=32, compressor=compressor, avg_period=avg_period)
    assert torch.isfinite(final).all()
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5]), losses


def test_one_worker_without_compression_is_momentum_sgd():
    """K = 1, C = identity: the same loop with torch's own group norm, clipping and SGD.  Every step rounds differently in
    both (sums of up to 32 * 1024 float32 terms, 2^-24 each), and three steps at lr 0.05 carry it on: 1e-4 of the update."""
    from paper_2008_05823_b200 import train_example as te
    steps, lr, top = 3, 0.05, 1.0
    torch.backends.cudnn.allow_tf32, keep = False, torch.backends.cudnn.allow_tf32
    try:
        losses, final = te.train(steps=steps, workers=1, blocks=1, classes=4, batch_size=16, lr=lr, compressor="identity",
                                 max_norm=top, amp=False, mode=sb.EF)
        torch.manual_seed(0)
        model = te.ResNetGN(1, 4).cuda().to(memory_format=torch.channels_last)
        start = torch.cat([p.detach().permute(0, 2, 3, 1).reshape(-1) if p.dim() == 4 else p.detach().reshape(-1) for p in model.parameters()])
        for m in model.modules():
            if isinstance(m, te.GroupNorm):
                def plain(x, residual=None, m=m):
                    z = torch.nn.functional.group_norm(x, m.num_groups, m.weight, m.bias, m.eps)
                    return torch.relu(z if residual is None else z + residual)
                m.forward = plain
        gen = torch.Generator(device="cuda").manual_seed(1)
        centers = torch.randn((4, 3, 32, 32), device="cuda", generator=gen)
        opt = torch.optim.SGD(model.parameters(), lr=lr, momentum=0.9)
        for i in range(steps):
            images, labels = te.batch(gen, centers, 16)
            loss = torch.nn.functional.cross_entropy(model(images), labels)
            opt.zero_grad()
            loss.backward()
            torch.nn.utils.clip_grad_norm_(model.parameters(), top)
            opt.step()
            assert abs(float(loss.detach()) - losses[i]) < 1e-3 * abs(losses[i])
    finally:
        torch.backends.cudnn.allow_tf32 = keep
    want = torch.cat([p.detach().permute(0, 2, 3, 1).reshape(-1) if p.dim() == 4 else p.detach().reshape(-1) for p in model.parameters()])
    assert float((final - want).norm()) < 1e-4 * float((want - start).norm())
