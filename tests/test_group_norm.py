"""Group norm with an activation, channels last: refusals (no GPU), and on the GPU forward and backward against the formulas
in float64, gradients against differences too.

Tolerances come with the reference, element by element, from u = 2^-24 and the number of roundings in sequence:
a statistic passes at most L = 16 + P / (4 max(1, 256 // C)) of them (runs of a thread's pixels, then a block's threads, then
the blocks), a gradient sum S = 32 + P / max(1, 256 // C) + N.  mean is then within L u mean|x|, var within
L u (2 + k) of itself with k = |mean| / std; x - mean, * rstd, * w, + b and the residual round once each.  A slope or
activation costs 16 u in float32; in 16 bits it uses the fast exponential, whose error is 2 + 1.2 |z| units: 128 u up to the
|z| < 40 that occur here.  relu's slope jumps at 0: where |z| is within its error, either value is right.  Outputs round once:
2^-24, 2^-8 (bfloat16), 2^-11 (float16) relative, half the smallest subnormal absolute."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2008_05823_b200 import binding as sb

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
ROUND = {F32: U, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}


# ---- refusals of the C entry points -----------------------------------------------------------------------------------

def desc(**kw):
    base = dict(type=0, param_type=0, activation=0, groups=4, samples=2, pixels=9, channels=8, x_sample=72, x_pixel=8,
                residual_sample=0, residual_pixel=0, dy_sample=72, dy_pixel=8, eps=1e-5)
    base.update(kw)
    return sb.SaeGroupNormDesc(**base)


BAD = [dict(type=3), dict(type=-1), dict(param_type=5), dict(activation=4), dict(activation=-1), dict(groups=0), dict(groups=3),
       dict(groups=16), dict(samples=-1), dict(samples=2 ** 24 + 1), dict(pixels=-1), dict(pixels=2 ** 30 + 1), dict(channels=0),
       dict(channels=2 ** 20 + 4), dict(eps=-1.0), dict(eps=math.nan), dict(x_pixel=-8), dict(dy_sample=-1), dict(residual_pixel=-1),
       dict(samples=2 ** 20, channels=2 ** 12, groups=2 ** 12)]


@pytest.mark.parametrize("kw", BAD)
def test_bad_descriptions_are_refused(kw):
    L, p = sb.lib(), C.c_void_p(256)          # never dereferenced: the checks fail first
    d = C.byref(desc(**kw))
    assert L.sae_group_norm_workspace(d, 0) == -1
    assert L.sae_group_norm_forward(d, p, None, p, p, p, p, p, p, 1 << 20, None) == sb.ERR_INVALID_ARG
    assert L.sae_group_norm_backward(d, p, p, None, p, p, p, p, p, None, p, p, p, 1 << 20, None) == sb.ERR_INVALID_ARG


def test_null_and_misaligned_pointers_are_refused():
    L, p, odd = sb.lib(), C.c_void_p(256), C.c_void_p(258)
    d = C.byref(desc())
    assert L.sae_group_norm_workspace(None, 1) == -1
    for i in (0, 4, 5, 6):
        args = [p, None, p, p, p, p, p, p]
        args[i] = None
        assert L.sae_group_norm_forward(d, *args, 1 << 20, None) == sb.ERR_INVALID_ARG, i
    for i in (0, 1, 2, 3, 4):
        args = [p, None, p, p, p, p, p, p]
        args[i] = odd
        assert L.sae_group_norm_forward(d, *args, 1 << 20, None) == sb.ERR_INVALID_ARG, i
    for i in (0, 1, 3, 4, 7):
        args = [p, p, None, p, p, p, p, p, None, p, p, p]
        args[i] = None
        assert L.sae_group_norm_backward(d, *args, 1 << 20, None) == sb.ERR_INVALID_ARG, i


# ---- the formulas in float64, with their tolerances ----------------------------------------------------------------------

def last(t):
    """[n, c, *space] -> float64 [n, pixels, c]."""
    a = t.detach().double().cpu().numpy()
    n, c = a.shape[:2]
    return np.moveaxis(a.reshape(n, c, -1), 1, 2)


def act64(z, act):
    erf = np.vectorize(math.erf, otypes=[np.float64])
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-z))
    phi, cdf = np.exp(-z * z / 2) / math.sqrt(2 * math.pi), 0.5 * (1 + erf(z / math.sqrt(2))) if z.size else z
    return {"none": (z, np.ones_like(z)), "relu": (np.maximum(z, 0), (z > 0) * 1.0), "silu": (z * s, s * (1 + z * (1 - s))),
            "gelu": (z * cdf, cdf + z * phi)}[act]


def spread(v, c):
    return np.repeat(v, c // v.shape[1], axis=1)[:, None, :]


def over_group(v, groups):
    """Sums of [n, p, c] over a group's channels and pixels: [n, groups]."""
    n, p, c = v.shape
    return v.reshape(n, p, groups, c // groups).sum((1, 3))


def act_cost(dtype):
    return 16 * U if dtype == F32 else 128 * U


def forward64(x, groups, w, b, eps, act, res, dtype):
    n, p, c = x.shape
    M = p * (c // groups)
    L = 16 + p / (4 * max(1, 256 // c))
    mean = over_group(x, groups) / M
    mean_tol = L * U * over_group(np.abs(x), groups) / M
    var = over_group((x - spread(mean, c)) ** 2, groups) / M
    k = np.sqrt(mean ** 2 / np.maximum(var, 1e-300))
    var_tol = L * U * (2 + k) * var + mean_tol ** 2
    rstd = 1 / np.sqrt(var + eps)
    rstd_rel = 0.5 * var_tol * rstd ** 2 + 2 * U
    xhat = (x - spread(mean, c)) * spread(rstd, c)
    xhat_tol = spread(mean_tol * rstd, c) + np.abs(xhat) * (spread(rstd_rel, c) + 2 * U)
    z = xhat * w + b + res
    z_tol = np.abs(w) * xhat_tol + 4 * U * (np.abs(xhat * w) + np.abs(b) + np.abs(res))
    y, _ = act64(z, act)
    y_tol = 1.2 * z_tol + (act_cost(dtype) * (1 + np.abs(z)) if act in ("silu", "gelu") else 0.0)
    y_tol = y_tol + (np.abs(y) + y_tol) * ROUND[dtype] + TINY[dtype]
    return (y, y_tol), (mean, mean_tol + U * np.abs(mean)), (rstd, rstd * (rstd_rel + U))


def backward64(dy, x, mean, rstd, groups, w, b, act, res, dtype):
    n, p, c = x.shape
    M = p * (c // groups)
    S = 32 + p / max(1, 256 // c) + n
    rs = spread(rstd, c)
    xhat = (x - spread(mean, c)) * rs
    z = xhat * w + b + res
    z_tol = 5 * U * (np.abs(xhat * w) + np.abs(b) + np.abs(res))
    _, slope = act64(z, act)
    dz = dy * slope
    if act == "relu":
        dz_tol = np.where(np.abs(z) <= z_tol, np.abs(dy), 0.0)
    elif act == "none":
        dz_tol = np.zeros_like(dz)
    else:
        dz_tol = np.abs(dy) * (z_tol + act_cost(dtype) * (1 + np.abs(z)))
    dzx, dzx_tol = dz * xhat, dz_tol * np.abs(xhat) + 3 * U * np.abs(dz * xhat)

    def summed(v, tol, over):
        return over(v), over(tol) + S * U * over(np.abs(v))

    channel = lambda v: v.sum((0, 1))  # noqa: E731
    db, dw = summed(dz, dz_tol, channel), summed(dzx, dzx_tol, channel)
    g, g_tol = dz * w, dz_tol * np.abs(w) + U * np.abs(dz * w)
    mg = summed(g, g_tol, lambda v: over_group(v, groups) / M)
    mx = summed(dzx * w, dzx_tol * np.abs(w) + U * np.abs(dzx * w), lambda v: over_group(v, groups) / M)
    dx = rs * (g - spread(mg[0], c) - xhat * spread(mx[0], c))
    inner = np.abs(g) + spread(np.abs(mg[0]), c) + np.abs(xhat) * spread(np.abs(mx[0]), c)
    dx_tol = rs * (g_tol + spread(mg[1], c) + np.abs(xhat) * spread(mx[1], c) + 6 * U * inner)
    dx_tol = dx_tol + (np.abs(dx) + dx_tol) * ROUND[dtype] + TINY[dtype]
    dz_tol = dz_tol + (np.abs(dz) + dz_tol) * ROUND[dtype] + TINY[dtype]
    return (dx, dx_tol), (dz, dz_tol), dw, db


def close(got, want, what):
    want, tol = want
    got = got if isinstance(got, np.ndarray) else got.detach().double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), got.size, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], np.broadcast_to(tol, got.shape)[bad][:3])


# ---- cases -----------------------------------------------------------------------------------------------------------------

def tensor(shape, dtype, gen, wide=0, offset=0, scale=1.0, shift=0.0):
    """[n, c, *space], channels last, `wide` unread channels beside the c, starting `offset` elements into its memory."""
    n, c, *space = shape
    t = (torch.randn((n, *space, c + wide), generator=gen) * scale + shift).to(dtype)
    if offset:
        flat = torch.empty(t.numel() + offset, dtype=dtype, device="cuda")
        held = flat[offset:].view(t.shape)
        held.copy_(t)
        t = held
    return t.cuda()[..., :c].movedim(-1, 1)


# (shape, groups, dtype, activation, residual, wide, offset, mean shift)
CASES = [
    ((1, 1, 1, 1), 1, F32, "none", False, 0, 0, 0.0),
    ((2, 8, 1, 1), 4, F32, "relu", False, 0, 0, 0.0),
    ((3, 6), 2, BF16, "silu", True, 0, 0, 0.0),
    ((1, 16, 32, 32), 4, BF16, "relu", False, 0, 0, 0.0),
    ((4, 16, 32, 32), 4, F32, "relu", True, 0, 0, 0.5),
    ((2, 64, 7, 9), 32, F16, "gelu", True, 0, 0, 0.2),
    ((2, 64, 14, 14), 32, BF16, "silu", False, 0, 0, 0.0),
    ((3, 90, 11, 13), 15, F32, "silu", False, 37, 0, 0.3),
    ((3, 90, 11, 13), 15, BF16, "gelu", True, 6, 0, 0.3),
    ((2, 48, 9, 10), 8, BF16, "relu", True, 0, 0, 0.0),          # 6 channels a group: vectors span groups
    ((2, 24, 31, 5), 24, F16, "silu", True, 0, 0, 0.1),          # one channel a group
    ((2, 40, 6, 6), 1, F32, "gelu", True, 0, 0, 0.0),            # one group
    ((2, 256, 12, 12), 32, BF16, "relu", True, 8, 0, 0.0),
    ((1, 2048, 7, 7), 32, F32, "none", True, 0, 0, 0.0),
    ((1, 3000, 3, 3), 3, BF16, "none", False, 0, 0, 0.0),
    ((2, 5000, 2), 5, F32, "relu", False, 0, 0, 0.0),
    ((5, 12, 3, 4, 5), 3, F16, "none", True, 0, 0, 0.0),         # three axes
    ((2, 32, 300), 8, F32, "silu", True, 0, 3, 0.0),             # nothing aligned beyond the element
    ((2, 32, 300), 8, BF16, "relu", True, 0, 5, 0.0),
    ((1, 32, 150, 151), 8, BF16, "relu", True, 0, 0, 0.0),       # long
    ((1, 4, 300, 301), 2, F32, "gelu", False, 0, 0, 0.0),
    ((2, 64, 64, 65), 2, F16, "relu", False, 0, 0, 0.0),
    ((70, 8, 5, 5), 2, BF16, "gelu", False, 0, 0, 0.0),
    ((2, 16, 10, 10), 4, F32, "none", False, 0, 0, 1000.0),      # mean far above the spread
    ((1, 130, 100, 100), 13, F32, "relu", True, 2, 0, 0.0),
    ((9, 64, 56, 56), 8, F32, "silu", True, 0, 0, 0.0),
    ((2, 128, 40, 40), 32, BF16, "silu", True, 0, 0, 0.0),
    # no multiple of a vector, without gaps: several pixels make a row (large enough for it), and beside them ones that do not
    ((8, 35, 104, 100), 7, BF16, "relu", True, 0, 0, 0.3),
    ((4, 90, 100, 60), 15, F16, "silu", False, 0, 0, 0.0),
    ((2, 99, 120, 100), 3, F32, "gelu", True, 0, 0, 0.2),
    ((3, 20, 200, 100), 20, BF16, "gelu", True, 0, 0, 0.0),
    ((1, 111, 199, 101), 37, BF16, "relu", False, 0, 0, 0.0),
    ((2, 35, 201, 200), 5, BF16, "none", True, 5, 0, 0.0),
    # groups wider than a block, and tensors too large for one pass: whole vectors in a group, and groups that cut them
    ((2, 4100, 2), 1, F32, "relu", True, 0, 0, 0.0),
    ((3, 9000, 5), 2, BF16, "silu", False, 0, 0, 0.2),
    ((4, 3000, 30, 31), 3, BF16, "relu", False, 0, 0, 0.0),
    ((7, 256, 56, 64), 32, BF16, "relu", True, 0, 0, 0.3),
    ((7, 256, 56, 64), 16, F16, "silu", False, 8, 0, 0.0),
    ((6, 128, 64, 64), 32, F32, "none", True, 0, 0, 0.0),
    ((6, 128, 64, 64), 8, F32, "silu", True, 4, 0, 0.1),
    ((3, 320, 100, 100), 32, BF16, "relu", True, 0, 0, 0.0),
]


def build(case, seed, param=F32):
    shape, groups, dtype, act, has_res, wide, offset, shift = case
    gen = torch.Generator().manual_seed(seed)
    c = shape[1]
    w = (1 + 0.3 * torch.randn(c, generator=gen)).to(param).cuda()
    b = (0.3 * torch.randn(c, generator=gen)).to(param).cuda()
    x = tensor(shape, dtype, gen, wide, offset, 1.0 + 0.5 * torch.rand(c + wide, generator=gen), shift)
    res = tensor(shape, dtype, gen, 0, offset) if has_res else None
    dy = tensor(shape, dtype, gen, wide, 0)
    return x, w, b, res, dy


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward_and_backward(case):
    from paper_2008_05823_b200 import group_norm as gn
    shape, groups, dtype, act, has_res, *_ = CASES[case]
    x, w, b, res, dy = build(CASES[case], case)
    wn, bn = w.double().cpu().numpy(), b.double().cpu().numpy()
    rn = last(res) if has_res else 0.0
    y, mean, rstd = gn.group_norm_forward(x, groups, w, b, 1e-5, act, res)
    assert y.shape == x.shape and y.dtype == x.dtype
    want_y, want_mean, want_rstd = forward64(last(x), groups, wn, bn, 1e-5, act, rn, dtype)
    close(mean, want_mean, "mean")
    close(rstd, want_rstd, "rstd")
    close(last(y), want_y, "y")
    dx, dres, dw, db = gn.group_norm_backward(dy, x, mean, rstd, groups, w, b, act, res)
    want_dx, want_dz, want_dw, want_db = backward64(last(dy), last(x), mean.double().cpu().numpy(), rstd.double().cpu().numpy(),
                                                    groups, wn, bn, act, rn, dtype)
    close(last(dx), want_dx, "dx")
    close(dw, want_dw, "dweight")
    close(db, want_db, "dbias")
    assert (dres is not None) == has_res
    if has_res:
        close(last(dres), want_dz, "dresidual")
    again = gn.group_norm_backward(dy, x, mean, rstd, groups, w, b, act, res)
    for p, q in zip((dx, dres, dw, db), again):
        assert p is None and q is None or torch.equal(p, q)


@pytest.mark.gpu
@pytest.mark.parametrize("param", [BF16, F16])
def test_parameters_of_16_bits_or_none(param):
    from paper_2008_05823_b200 import group_norm as gn
    case = ((2, 32, 8, 8), 4, BF16, "silu", False, 0, 0, 0.0)
    x, w, b, _, dy = build(case, 50, param)
    wn, bn = w.double().cpu().numpy(), b.double().cpu().numpy()
    y, mean, rstd = gn.group_norm_forward(x, 4, w, b, 1e-5, "silu")
    close(last(y), forward64(last(x), 4, wn, bn, 1e-5, "silu", 0.0, BF16)[0], "y")
    dx, _, dw, db = gn.group_norm_backward(dy, x, mean, rstd, 4, w, b, "silu")
    m, r = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
    want_dx, _, want_dw, want_db = backward64(last(dy), last(x), m, r, 4, wn, bn, "silu", 0.0, BF16)
    assert dw.dtype == param
    close(last(dx), want_dx, "dx")
    for got, (want, tol) in ((dw, want_dw), (db, want_db)):
        close(got, (want, tol + (np.abs(want) + tol) * ROUND[param] + TINY[param]), "parameter gradient")
    for w1, b1 in ((None, None), (w, None), (None, b)):
        wn1 = np.ones(32) if w1 is None else wn
        bn1 = np.zeros(32) if b1 is None else bn
        y, mean, rstd = gn.group_norm_forward(x, 4, w1, b1, 1e-5, "silu")
        close(last(y), forward64(last(x), 4, wn1, bn1, 1e-5, "silu", 0.0, BF16)[0], "y")
        dx, _, dw, db = gn.group_norm_backward(dy, x, mean, rstd, 4, w1, b1, "silu")
        close(last(dx), backward64(last(dy), last(x), m, r, 4, wn1, bn1, "silu", 0.0, BF16)[0], "dx")
        assert (dw is None) == (w1 is None) and (db is None) == (b1 is None)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("shape,groups", [((2, 12, 5, 7), 4), ((1, 64, 9, 9), 8), ((3, 16, 40), 2)])
def test_gradients_against_differences(shape, groups, act):
    """<gradient, v> against the central difference of sum(r * y) along v, every input at once.  The difference at h / 2 is
    off by a third of what it moved from the one at h, and by the outputs' roundings (40 u |r y|, with the statistics') / h."""
    from paper_2008_05823_b200 import group_norm as gn
    gen = torch.Generator().manual_seed(9)
    ins = [tensor(shape, F32, gen), (1 + 0.2 * torch.randn(shape[1], generator=gen)).cuda(), torch.randn(shape[1], generator=gen).cuda(),
           tensor(shape, F32, gen)]
    r = tensor(shape, F32, gen)
    vs = [torch.randn(t.shape, generator=gen).cuda() for t in ins]
    leaves = [t.clone().requires_grad_() for t in ins]
    y = gn.group_norm(leaves[0], groups, leaves[1], leaves[2], 1e-5, act, leaves[3])
    (y * r).sum().backward()

    def loss(h):
        moved = [t + h * v for t, v in zip(ins, vs)]
        y = gn.group_norm_forward(moved[0], groups, moved[1], moved[2], 1e-5, act, moved[3])[0]
        return float((y.double() * r.double()).sum())

    h = 2.0 ** -5
    big, small = (loss(h) - loss(-h)) / (2 * h), (loss(h / 2) - loss(-h / 2)) / h
    analytic = sum(float((t.grad.double() * v.double()).sum()) for t, v in zip(leaves, vs))
    noise = 40 * U * float((y.detach().double().abs() * r.double().abs() + r.double().abs()).sum()) / h
    assert abs(analytic - small) <= abs(big - small) + noise, (analytic, big, small, noise)


@pytest.mark.gpu
def test_module_and_autograd():
    from paper_2008_05823_b200 import group_norm as gn
    torch.manual_seed(0)
    m = gn.GroupNorm(4, 16, activation="relu", device="cuda")
    with torch.no_grad():
        m.weight.uniform_(0.5, 1.5)
        m.bias.normal_()
    x = torch.randn(3, 16, 6, 5, device="cuda").to(memory_format=torch.channels_last).requires_grad_()
    res = torch.randn(3, 16, 6, 5, device="cuda").to(memory_format=torch.channels_last).requires_grad_()
    out = m(x, res)
    assert out.is_contiguous(memory_format=torch.channels_last)
    ref = torch.relu(torch.nn.functional.group_norm(x.double(), 4, m.weight.double(), m.bias.double(), 1e-5) + res.double())
    assert torch.allclose(out.double(), ref, atol=1e-5)
    dy = torch.randn_like(out)
    for grad in (dy, dy.contiguous(), torch.ones(1, device="cuda").expand(3, 16, 6, 5)):   # any order, broadcast too
        got = torch.autograd.grad(out, [x, m.weight, m.bias, res], grad, retain_graph=True)
        want = torch.autograd.grad(ref, [x, m.weight, m.bias, res], grad.double(), retain_graph=True)
        for a, b in zip(got, want):
            assert torch.allclose(a.double(), b.double(), atol=1e-4), float((a - b).abs().max())
    # a residual shared by the samples: its gradient is summed by the expansion's own
    one = torch.randn(1, 16, 6, 5, device="cuda").to(memory_format=torch.channels_last).requires_grad_()
    plain = gn.GroupNorm(4, 16, device="cuda")
    (plain(x, one.expand(3, 16, 6, 5)) * dy).sum().backward()
    assert torch.allclose(one.grad, dy.sum(0, keepdim=True), atol=1e-5)
    # no pixels: [n, c], its gradient broadcast
    flat = torch.randn(3, 16, device="cuda", requires_grad=True)
    m(flat).sum().backward()
    ref = torch.relu(torch.nn.functional.group_norm(flat.double(), 4, m.weight.double(), m.bias.double(), 1e-5))
    assert torch.allclose(flat.grad.double(), torch.autograd.grad(ref.sum(), [flat])[0].double(), atol=1e-4)
    frozen = gn.group_norm(x, 4, m.weight.detach(), m.bias.detach(), 1e-5, "silu")
    (gx,) = torch.autograd.grad(frozen, [x], dy)
    assert torch.isfinite(gx).all()


@pytest.mark.gpu
def test_empty_and_constant_and_nan():
    from paper_2008_05823_b200 import group_norm as gn
    w, b = torch.ones(8, device="cuda"), torch.full((8,), 0.25, device="cuda")
    for shape in ((0, 8, 4, 4), (2, 8, 0, 4)):
        x = torch.empty(shape, device="cuda")
        y, mean, rstd = gn.group_norm_forward(x, 2, w, b)
        assert y.shape == x.shape and mean.shape == (shape[0], 2) and torch.isnan(mean).all()
        dx, _, dw, db = gn.group_norm_backward(x, x, mean, rstd, 2, w, b)
        assert dx.shape == x.shape and not dw.any() and not db.any()
    flat = torch.full((2, 8, 5, 5), 3.0, device="cuda").to(memory_format=torch.channels_last)
    y, mean, rstd = gn.group_norm_forward(flat, 2, w, b, 1e-5)
    assert (y == 0.25).all() and (mean == 3).all()
    y, _, _ = gn.group_norm_forward(flat, 2, w, b, 0.0)                     # 0 * inf
    assert torch.isnan(y).all()
    x = torch.randn(2, 8, 5, 5, device="cuda").to(memory_format=torch.channels_last)
    x[1, 2, 3, 3] = math.nan
    x[0, 7, 0, 0] = math.inf
    for act in gn.ACT_OF:
        y, _, _ = gn.group_norm_forward(x, 2, w, b, 1e-5, act)
        assert torch.isnan(y[1, :4]).all() and torch.isfinite(y[1, 4:]).all() and torch.isfinite(y[0, :4]).all()
        assert torch.isnan(y[0, 7, 0, 0])
    big = (torch.randn(1, 8, 6, 6, device="cuda") * 1e18).to(memory_format=torch.channels_last)
    y, _, _ = gn.group_norm_forward(big, 2, w, b)
    assert torch.isfinite(y).all() and 0.5 < float((y - 0.25).std()) < 1.5


@pytest.mark.gpu
def test_streams_capture_and_same_bits():
    from paper_2008_05823_b200 import group_norm as gn
    x, w, b, res, dy = build(CASES[12], 77)
    want = gn.group_norm_forward(x, 32, w, b, 1e-5, "relu", res)
    want_b = gn.group_norm_backward(dy, x, want[1], want[2], 32, w, b, "relu", res)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = gn.group_norm_forward(x, 32, w, b, 1e-5, "relu", res)
        got_b = gn.group_norm_backward(dy, x, got[1], got[2], 32, w, b, "relu", res)
    side.synchronize()
    for p, q in zip((*want, *want_b), (*got, *got_b)):
        assert torch.equal(p, q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = gn.group_norm_forward(x, 32, w, b, 1e-5, "relu", res)
        got_b = gn.group_norm_backward(dy, x, got[1], got[2], 32, w, b, "relu", res)
    for t in (*got, *got_b):
        t.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for p, q in zip((*want, *want_b), (*got, *got_b)):
        assert torch.equal(p, q)


@pytest.mark.gpu
def test_a_sample_past_31_bits():
    """More than 2^31 elements a sample: every part is normalised, and the last pixel lands in its place."""
    from paper_2008_05823_b200 import group_norm as gn
    p, c = 2 ** 25 + 3, 64
    x = torch.zeros((1, p, c), device="cuda", dtype=BF16)
    x[0, ::2] = 2.0
    x = x.movedim(-1, 1)
    y, mean, rstd = gn.group_norm_forward(x, 4, None, None, 0.0)
    share = ((p + 1) // 2) / p
    assert torch.allclose(mean.double(), torch.tensor(2 * share, dtype=torch.float64, device="cuda"), rtol=1e-6, atol=0)
    assert bool((y[0, :, -1] == 1).all()) and bool((y[0, :, 2 ** 25 - 1] == -1).all())
    assert int((y == 1).sum()) == ((p + 1) // 2) * c


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(40000, 8, 1, 3), (40000, 64, 3, 3)])
def test_more_samples_than_a_grid_dimension(shape):
    from paper_2008_05823_b200 import group_norm as gn
    n, c = shape[:2]
    case = (shape, 2, BF16, "relu", False, 0, 0, 0.3)
    x, w, b, _, dy = build(case, 5)
    y, mean, rstd = gn.group_norm_forward(x, 2, w, b, 1e-5, "relu")
    dx, _, dw, db = gn.group_norm_backward(dy, x, mean, rstd, 2, w, b, "relu")
    some = [0, 1, 32767, 32768, 32769, n - 1]
    wn, bn = w.double().cpu().numpy(), b.double().cpu().numpy()
    want_y, want_mean, _ = forward64(last(x[some]), 2, wn, bn, 1e-5, "relu", 0.0, BF16)
    close(last(y[some]), want_y, "y")
    close(mean[some], want_mean, "mean")
    m, r = mean.double().cpu().numpy(), rstd.double().cpu().numpy()
    want_dx, _, want_dw, want_db = backward64(last(dy), last(x), m, r, 2, wn, bn, "relu", 0.0, BF16)
    close(last(dx), want_dx, "dx")
    close(dw, want_dw, "dweight")
    close(db, want_db, "dbias")


@pytest.mark.gpu
def test_python_refusals():
    from paper_2008_05823_b200 import group_norm as gn
    x = torch.randn(2, 8, 4, 4, device="cuda").to(memory_format=torch.channels_last)
    w = torch.ones(8, device="cuda")
    bad = [(x.cpu(), 2, None, {}), (x.double(), 2, None, {}), (x, 3, None, {}), (x, 0, None, {}), (x.contiguous(), 2, None, {}), (x[:, ::2], 2, None, {}),
           (x[:, :, :, ::2].expand(2, 8, 4, 2)[:, :, :3], 2, None, {"activation": "tanh"}), (x, 2, w[:4], {}), (x, 2, w.cpu(), {}),
           (x, 2, torch.ones(16, device="cuda")[::2], {}), (x, 2, w, {"bias": w.bfloat16()}), (x, 2, w, {"residual": x[:1]}),
           (x, 2, w, {"residual": x.bfloat16()}), (x, 2, w, {"residual": x.contiguous()}), (x[:, :, ::2, ::3], 2, None, {})]
    for t, groups, weight, kw in bad:
        with pytest.raises(ValueError):
            gn.group_norm_forward(t, groups, weight, **kw)
    with pytest.raises(sb.SaeError):
        gn.group_norm_forward(x, 2, w, eps=-1.0)
    y, mean, rstd = gn.group_norm_forward(x, 2, w)
    for args in ((x[:1], x, mean, rstd), (x, x, mean[:1], rstd), (x, x, mean, rstd.double()), (x, x, mean.t(), rstd)):
        with pytest.raises(ValueError):
            gn.group_norm_backward(*args, 2, w)
    for kw in ((3, 8), (0, 8)):
        with pytest.raises(ValueError):
            gn.GroupNorm(*kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shape,groups,wide", [((2, 35, 201, 200), 5, 5), ((9, 33, 130, 131), 3, 0), ((70, 130, 30, 31), 13, 1)])
def test_second_pass_reads_what_the_first_has_written(shape, groups, wide, dtype):
    """Two passes over single 16-bit elements: with a residual the second one reads dresidual, without it dy.  Where there is no
    activation both are the same values, so dx has the same bits, whatever was in dresidual's memory before."""
    from paper_2008_05823_b200 import group_norm as gn
    x, w, b, res, dy = build((shape, groups, dtype, "none", True, wide, 0, 0.1), 21)
    _, mean, rstd = gn.group_norm_forward(x, groups, w, b)
    want, none, dw, db = gn.group_norm_backward(dy, x, mean, rstd, groups, w, b)
    assert none is None
    for fill in (math.nan, 1.0, 1.0, 1.0):
        junk = [torch.full_like(x, fill) for _ in range(3)]
        del junk                                     # the next call's outputs lie there
        dx, dres, dw2, db2 = gn.group_norm_backward(dy, x, mean, rstd, groups, w, b, "none", res)
        assert torch.equal(dx, want) and torch.equal(dres, dy) and torch.equal(dw, dw2) and torch.equal(db, db2)


# ---- z's roundings: no tolerance ---------------------------------------------------------------------------------------------

def plain_z(x, mean, rstd, w, b, res, groups):
    """x - mean, * rstd, * w, + b, + residual, one float32 operation after the other, pixels before channels."""
    c = x.shape[1]
    at = lambda s: s.repeat_interleave(c // groups, 1).view(x.shape[0], *[1] * (x.dim() - 2), c)  # noqa: E731
    z = (x.movedim(1, -1).float() - at(mean)) * at(rstd)
    z = z * w + b
    return z if res is None else z + res.movedim(1, -1).float()


# (shape, groups, unread channels beside x): one pass and two, vectors of 16 bytes, of two elements and of one, rows of pixels
Z_CASES = [((32, 256, 56, 56), 32, 0), ((128, 16, 32, 32), 4, 0), ((16, 256, 56, 56), 16, 2), ((16, 256, 56, 56), 256, 1), ((8, 35, 100, 100), 7, 0),
           ((2, 64, 14, 14), 32, 0), ((2, 30, 9, 11), 5, 0), ((2, 30, 9, 11), 5, 3), ((2, 35, 9, 11), 5, 0), ((1, 2048, 7, 7), 32, 0), ((40, 24), 3, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("has_res", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("case", range(len(Z_CASES)))
def test_every_step_of_z_is_rounded(case, dtype, has_res):
    """With the call's own statistics, y without an activation has the bits of the single operations; relu's mask in the
    backward call is z > 0, also where the two calls read x in different layouts."""
    from paper_2008_05823_b200 import group_norm as gn
    shape, groups, wide = Z_CASES[case]
    gen = torch.Generator(device="cuda").manual_seed(case)
    n, c, *space = shape

    def draw(beside):
        return torch.randn((n, *space, c + beside), device="cuda", generator=gen).to(dtype)[..., :c].movedim(-1, 1)

    x, res = draw(wide), draw(0).clamp(min=0) if has_res else None
    w, b = 1 + 0.1 * torch.randn(c, device="cuda", generator=gen), 0.1 * torch.randn(c, device="cuda", generator=gen)
    y, mean, rstd = gn.group_norm_forward(x, groups, w, b, 1e-5, "none", res)
    z = plain_z(x, mean, rstd, w, b, res, groups)
    assert torch.equal(y.movedim(1, -1), z.to(dtype))
    y, _, _ = gn.group_norm_forward(x, groups, w, b, 1e-5, "relu", res)
    assert torch.equal(y.movedim(1, -1), z.clamp(min=0).to(dtype))
    # dy = 1: dz is the mask, dbias counts it (exactly: fewer than 2^24 a channel)
    dense = x.movedim(1, -1).contiguous().movedim(-1, 1)
    ones = torch.ones_like(dense)
    for at in (x, dense):
        _, dres, _, db = gn.group_norm_backward(ones, at, mean, rstd, groups, w, b, "relu", res)
        assert torch.equal(db, (z > 0).sum(tuple(range(z.dim() - 1))).float())
        if has_res:
            assert torch.equal(dres.movedim(1, -1), (z > 0).to(dtype))


# Two passes, tiles that share groups and touch different numbers of them, many runs of pixels
TILED = [((1, 1152, 60, 60), 9, F32, 1), ((1, 2040, 1000), 85, F32, 1), ((2, 990, 3000), 99, F32, 1), ((1, 2560, 4000), 2, F32, 0), ((2, 2040, 1500), 85, BF16, 1),
         ((1, 5000, 900), 5, F16, 0), ((1, 4104, 1000), 2, BF16, 0)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(TILED)))
def test_tiles_that_share_a_group_agree(case):
    """Every tile normalises with the statistics that the call returns (y without an activation has the bits that those give),
    and they are the same bits on every call, forwards and backwards."""
    from paper_2008_05823_b200 import group_norm as gn
    shape, groups, dtype, wide = TILED[case]
    x, w, b, _, dy = build((shape, groups, dtype, "none", False, wide, 0, 0.7), 31 + case)
    y, mean, rstd = gn.group_norm_forward(x, groups, w, b)
    assert torch.equal(y.movedim(1, -1), plain_z(x, mean, rstd, w, b, None, groups).to(dtype))
    want_y, want_mean, want_rstd = forward64(last(x), groups, w.double().cpu().numpy(), b.double().cpu().numpy(), 1e-5, "none", 0.0, dtype)
    close(mean, want_mean, "mean")
    close(rstd, want_rstd, "rstd")
    back = gn.group_norm_backward(dy, x, mean, rstd, groups, w, b)
    for _ in range(30):
        again = gn.group_norm_forward(x, groups, w, b)
        assert all(torch.equal(p, q) for p, q in zip((y, mean, rstd), again))
        more = gn.group_norm_backward(dy, x, mean, rstd, groups, w, b)
        assert all(torch.equal(p, q) for p, q in zip(back, more) if p is not None)


# ---- long sums -------------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("n,c,pixels", [(230, 250, 16384), (65536, 8, 4), (230, 256, 8192)])
def test_long_sums_of_one_sign(n, c, pixels):
    """dy = 0.1 everywhere: each addition to a long chain rounds the same way, so a chain of k is off by up to k u (one of 16384: 2590 u).
    Here at most 128 + pixels / 32 of them follow one another in a thread, then 256 in a block and few more, and samples are
    added in double.  dweight: the same chains over terms of both signs."""
    from paper_2008_05823_b200 import group_norm as gn
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = (torch.randn((1, pixels, c), device="cuda", generator=gen) + 1).expand(n, pixels, c).movedim(-1, 1)
    dy = torch.full((1, 1, c), 0.1, device="cuda").expand(n, pixels, c).movedim(-1, 1)
    mean, rstd = torch.zeros(n, 2, device="cuda"), torch.ones(n, 2, device="cuda")
    _, _, dw, db = gn.group_norm_backward(dy, x, mean, rstd, 2, torch.ones(c, device="cuda"), torch.zeros(c, device="cuda"))
    depth = 128 + pixels / 32 + 16 if pixels > 1000 else pixels + 16
    tenth = float(torch.tensor(0.1))
    assert float((db.double() / (n * pixels * tenth) - 1).abs().max()) <= depth * U
    one = x[0].double()
    assert bool(((dw.double() - tenth * n * one.sum(1)).abs() <= (depth + 1) * U * tenth * n * one.abs().sum(1)).all())


# ---- activations over their whole range -------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations_over_their_range(act, dtype):
    """With weight 0, z is the bias.  y is act(z) rounded once: half a unit of the type, and the arithmetic's relative error: 16 u in
    float32 (and u z^2 from an exponential's argument), 24 u + 4 u z^2 in 16 bits (ex2 and rcp 4 u, the tail's polynomial 8 u, products;
    the exponent is rounded twice).  gelu in float32 is 1 + erf, whose error (two units of erf, one of its argument) is absolute.
    dbias sums the slope over 64 pixels: the same error of each of its two terms, and of 64 additions."""
    from paper_2008_05823_b200 import group_norm as gn
    c, p = 4096, 64
    z = np.linspace(-12.0, 12.0, c).astype(np.float32).astype(np.float64)
    b = torch.tensor(z, dtype=F32, device="cuda")
    x = torch.randn(1, p, c, device="cuda").to(dtype).movedim(-1, 1)
    w = torch.zeros(c, device="cuda")
    y, mean, rstd = gn.group_norm_forward(x, 32, w, b, 1e-5, act)
    erfc = np.array([math.erfc(-v / math.sqrt(2)) for v in z])
    cdf = 0.5 * erfc if act == "gelu" else 1 / (1 + np.exp(-z))
    rel = (16 * U + U * z ** 2) if dtype == F32 else (24 * U + 4 * U * z ** 2)
    off = 3 * U * np.abs(z) if dtype == F32 and act == "gelu" else 0.0
    want = z * cdf
    tol = np.abs(want) * (rel + ROUND[dtype]) * (1 + ROUND[dtype]) + off + TINY[dtype]
    close(last(y), (np.broadcast_to(want, (1, p, c)), np.broadcast_to(tol, (1, p, c))), "y")
    ones = torch.ones_like(x)
    _, _, _, db = gn.group_norm_backward(ones, x, mean, rstd, 32, w, b, act)
    other = z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi) if act == "gelu" else z * cdf * (1 - cdf)
    tol = p * ((np.abs(cdf) + np.abs(other)) * (rel + 80 * U) + (3 * U if dtype == F32 and act == "gelu" else 0.0))
    if act == "silu":
        tol = tol + p * cdf * np.abs(z) * 8 * U          # 1 - s loses the digits of s
    close(db, (p * (cdf + other), tol), "dbias")
