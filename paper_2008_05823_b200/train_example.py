"""A whole training loop on the library: a CIFAR-shaped ResNet with group norm, or a transformer encoder on masked tokens, K
simulated workers, clipped gradients.

Each iteration of Algorithm 1, for each worker k:
  x - e^(k) into the model's tensors    Sae.get_step_ahead, GradSet.unpack
  loss and gradients on its own batch   ResNet: conv + group_norm (with the shortcut and relu fused), torch autograd
                                        encoder: linear_cross_entropy over the vocabulary, of the positions that are masked
  (encoder, --orthogonal)               the gradients of the layers' matrices made orthogonal (Orthogonalizer)
  the gradients into row k              GradSet.pack (norm over all tensors, clipping, concatenation)
then one Sae.step.  Synthetic data: a fixed random image a class, plus noise; sequences that count up in steps of their own.

Usage: python -m paper_2008_05823_b200.train_example [--model resnet|encoder] [--steps 30] [--workers 4] [--blocks 3] [--layers 2]
       [--compressor sign|topk|identity] [--orthogonal]
"""
import argparse

import torch
from torch import nn
from torch.nn import functional as F

from . import binding, configs
from .cross_entropy import linear_cross_entropy
from .grads import GradSet
from .group_norm import GroupNorm
from .orthogonal import Orthogonalizer

COMPRESSORS = {"identity": binding.IDENTITY, "sign": binding.SIGN, "topk": binding.TOPK}


class Block(nn.Module):
    def __init__(self, cin, cout, groups):
        super().__init__()
        self.stride = 1 if cin == cout else 2
        self.conv1 = nn.Conv2d(cin, cout, 3, self.stride, 1, bias=False)
        self.norm1 = GroupNorm(groups, cout, activation="relu")
        self.conv2 = nn.Conv2d(cout, cout, 3, 1, 1, bias=False)
        self.norm2 = GroupNorm(groups, cout, activation="relu")

    def forward(self, x):
        shortcut = x
        if self.stride == 2:                    # parameter-free: every other pixel, new channels zero
            shortcut = F.pad(x[:, :, ::2, ::2], (0, 0, 0, 0, 0, x.shape[1])).contiguous(memory_format=torch.channels_last)
        return self.norm2(self.conv2(self.norm1(self.conv1(x))), shortcut)


class ResNetGN(nn.Module):
    """ResNet-(6 blocks + 2) for 32x32 images: the parameter list of configs.resnet_cifar_sizes, a group norm for each batch norm."""

    def __init__(self, blocks=3, classes=10, groups=4):
        super().__init__()
        self.conv = nn.Conv2d(3, 16, 3, 1, 1, bias=False)
        self.norm = GroupNorm(groups, 16, activation="relu")
        widths = [16] + [c for c in (16, 32, 64) for _ in range(blocks)]
        self.blocks = nn.Sequential(*[Block(a, b, groups) for a, b in zip(widths, widths[1:])])
        self.fc = nn.Linear(64, classes)

    def forward(self, x):
        return self.fc(self.blocks(self.norm(self.conv(x))).mean((2, 3)))


def batch(gen, centers, size):
    labels = torch.randint(len(centers), (size,), device="cuda", generator=gen)
    images = centers[labels] + torch.randn((size, 3, 32, 32), device="cuda", generator=gen)
    return images.contiguous(memory_format=torch.channels_last), labels


def train(steps=30, workers=4, blocks=3, classes=10, batch_size=32, lr=0.05, momentum=0.9, compressor="sign", max_norm=5.0,
          avg_period=0, seed=0, amp=True, mode=binding.SAEF):
    """Runs the loop; returns (the mean loss of every step, the final parameters as one vector)."""
    torch.manual_seed(seed)
    model = ResNetGN(blocks, classes).cuda().to(memory_format=torch.channels_last)
    params = list(model.parameters())
    sizes = [p.numel() for p in params]
    assert sizes == configs.resnet_cifar_sizes(blocks, classes)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    centers = torch.randn((classes, 3, 32, 32), device="cuda", generator=gen)

    one = GradSet.like(params)                              # a worker's tensors, as they lie in memory
    x0, _ = one.pack([p.detach() for p in params])
    sae = binding.Sae(workers, sizes, x0[0], compressor=COMPRESSORS[compressor], momentum=momentum, avg_period=avg_period,
                      topk_num=5, topk_den=100, mode=mode)
    grads, ahead = torch.empty(workers, one.d, device="cuda"), torch.empty(one.d, device="cuda")
    losses = []
    for _ in range(steps):
        total = 0.0
        for k in range(workers):
            one.unpack(sae.get_step_ahead(k, ahead), [p.detach() for p in params])
            images, labels = batch(gen, centers, batch_size)
            with torch.autocast("cuda", torch.bfloat16, enabled=amp):
                loss = F.cross_entropy(model(images), labels)
            model.zero_grad(set_to_none=True)
            loss.backward()
            one.pack([p.grad for p in params], grads[k], max_norm=max_norm)
            total = total + loss.detach()
        sae.step(grads, lr)
        losses.append(total / workers)
    sae.sync()
    final = sae.get_params()
    sae.close()
    one.close()
    return torch.stack(losses).tolist(), final


class EncoderLayer(nn.Module):
    def __init__(self, hidden, heads):
        super().__init__()
        self.heads = heads
        self.query, self.key, self.value, self.out = (nn.Linear(hidden, hidden) for _ in range(4))
        self.norm1 = nn.LayerNorm(hidden)
        self.up, self.down = nn.Linear(hidden, 4 * hidden), nn.Linear(4 * hidden, hidden)
        self.norm2 = nn.LayerNorm(hidden)

    def forward(self, x):
        q, k, v = (f(x).unflatten(-1, (self.heads, -1)).transpose(1, 2) for f in (self.query, self.key, self.value))
        x = self.norm1(x + self.out(F.scaled_dot_product_attention(q, k, v).transpose(1, 2).flatten(2)))
        return self.norm2(x + self.down(F.gelu(self.up(x))))


class Encoder(nn.Module):
    """The parameter list of configs.encoder_sizes, in its order; the output layer's weights are the word embedding's."""

    def __init__(self, layers, hidden, vocab, positions, heads):
        super().__init__()
        self.word, self.position, self.kind = nn.Embedding(vocab, hidden), nn.Embedding(positions, hidden), nn.Embedding(2, hidden)
        for e in (self.word, self.position, self.kind):
            nn.init.normal_(e.weight, std=hidden ** -0.5)
        self.norm = nn.LayerNorm(hidden)
        self.layers = nn.Sequential(*[EncoderLayer(hidden, heads) for _ in range(layers)])
        self.last = nn.Linear(hidden, hidden)

    def matrices(self):
        """The layers' matrices: what is made orthogonal."""
        return [p for p in self.layers.parameters() if p.dim() == 2]

    def forward(self, tokens, target):
        """The mean loss of the positions whose target is not -100."""
        x = self.word(tokens) + self.position.weight[:tokens.shape[1]] + self.kind.weight[0]
        x = torch.tanh(self.last(self.layers(self.norm(x))))
        return linear_cross_entropy(x, self.word.weight, target)


def masked_batch(gen, vocab, size, length, share=0.15):
    """Sequences start + i * step (mod vocab - 1); token vocab - 1 stands where a token is masked, and only there is a target."""
    start, step = (torch.randint(1, n, (size, 1), device="cuda", generator=gen) for n in (vocab - 1, 8))
    tokens = (start + step * torch.arange(length, device="cuda")) % (vocab - 1)
    masked = torch.rand((size, length), device="cuda", generator=gen) < share
    masked[:, 0] = True                         # a batch without any target has no mean
    return torch.where(masked, vocab - 1, tokens), torch.where(masked, tokens, -100)


def train_encoder(steps=30, workers=4, layers=2, hidden=64, vocab=1000, positions=64, heads=4, batch_size=16, length=48, lr=0.05, momentum=0.9,
                  compressor="sign", max_norm=1.0, avg_period=0, seed=0, amp=True, mode=binding.SAEF, orthogonal=False, scale=0.02):
    """Runs the loop; returns (the mean loss of every step, the final parameters as one vector).  orthogonal: the gradient of every matrix of
    the layers is replaced by `scale` times its orthogonal factor before clipping."""
    torch.manual_seed(seed)
    model = Encoder(layers, hidden, vocab, positions, heads).cuda()
    params, matrices = list(model.parameters()), model.matrices()
    sizes = [p.numel() for p in params]
    assert sizes == configs.encoder_sizes(layers, hidden, 4 * hidden, vocab, positions)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)

    one = GradSet.like(params)
    x0, _ = one.pack([p.detach() for p in params])
    plan = Orthogonalizer.like(matrices) if orthogonal else None
    sae = binding.Sae(workers, sizes, x0[0], compressor=COMPRESSORS[compressor], momentum=momentum, avg_period=avg_period,
                      topk_num=5, topk_den=100, mode=mode)
    grads, ahead = torch.empty(workers, one.d, device="cuda"), torch.empty(one.d, device="cuda")
    losses = []
    for _ in range(steps):
        total = 0.0
        for k in range(workers):
            one.unpack(sae.get_step_ahead(k, ahead), [p.detach() for p in params])
            tokens, target = masked_batch(gen, vocab, batch_size, length)
            with torch.autocast("cuda", torch.bfloat16, enabled=amp):
                loss = model(tokens, target)
            model.zero_grad(set_to_none=True)
            loss.backward()
            if plan:
                made = [p.grad for p in matrices]
                torch._foreach_mul_(plan(made, made), scale)
            one.pack([p.grad for p in params], grads[k], max_norm=max_norm)
            total = total + loss.detach()
        sae.step(grads, lr)
        losses.append(total / workers)
    sae.sync()
    final = sae.get_params()
    sae.close()
    one.close()
    if plan:
        plan.close()
    return torch.stack(losses).tolist(), final


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--compressor", choices=sorted(COMPRESSORS), default="sign")
    ap.add_argument("--model", choices=("resnet", "encoder"), default="resnet")
    ap.add_argument("--layers", type=int, default=2, help="of the encoder")
    ap.add_argument("--orthogonal", action="store_true", help="encoder: the gradients of the layers' matrices are made orthogonal")
    a = ap.parse_args()
    if a.orthogonal and a.model != "encoder":
        ap.error("--orthogonal goes with --model encoder")
    if a.model == "encoder":
        losses, _ = train_encoder(a.steps, a.workers, a.layers, compressor=a.compressor, orthogonal=a.orthogonal)
    else:
        losses, _ = train(a.steps, a.workers, a.blocks, compressor=a.compressor)
    for i, v in enumerate(losses):
        print(f"step {i + 1}: loss {v:.4f}")


if __name__ == "__main__":
    main()
