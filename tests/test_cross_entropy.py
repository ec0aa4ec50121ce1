"""Linear cross entropy against the definition in float64: values, gradients, rows without a target, targets that are none, masks by
the bias, infinities, layouts, streams, captured graphs, refusals."""
import ctypes as C
import math

import pytest
import torch

from paper_2008_05823_b200 import binding as sb
from paper_2008_05823_b200 import cross_entropy as ce

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
IGNORE = -100


# ---- refusals, without a GPU --------------------------------------------------------------------------------------------------

def desc(**kw):
    base = dict(type=sb.TYPE_BFLOAT, bias_type=sb.TYPE_FLOAT, reduction=sb.REDUCE_MEAN, has_bias=0, rows=4, features=8, classes=5,
                x_pitch=8, weight_pitch=8, ignore_index=-100)
    return sb.SaeLinearCeDesc(**(base | kw))


@pytest.mark.parametrize("bad", [dict(type=3), dict(type=-1), dict(bias_type=7, has_bias=1), dict(reduction=3), dict(rows=-1), dict(rows=(1 << 24) + 1),
                                 dict(features=0), dict(features=(1 << 17) + 1, x_pitch=1 << 18, weight_pitch=1 << 18), dict(classes=0),
                                 dict(classes=(1 << 24) + 1), dict(x_pitch=7), dict(weight_pitch=7)])
def test_bad_descriptions_are_refused(bad):
    L, p = sb.lib(), C.c_void_p(256)                       # never dereferenced
    d = desc(**bad)
    assert L.sae_linear_ce_workspace(C.byref(d), p, 0) == -1
    assert L.sae_linear_ce_forward(C.byref(d), p, p, None, p, p, p, p, p, 1 << 30, None) == sb.ERR_INVALID_ARG
    assert L.sae_linear_ce_backward(C.byref(d), p, p, p, None, p, p, p, p, p, None, p, 1 << 30, None) == sb.ERR_INVALID_ARG


def test_null_and_misaligned_pointers_are_refused():
    L, p, odd = sb.lib(), C.c_void_p(256), C.c_void_p(257)
    d, withbias = desc(), desc(has_bias=1)
    good = [p, p, None, p, p, p, p, p]
    for i in (0, 1, 3, 4, 5, 6, 7):
        for v in (None, odd):
            args = list(good)
            args[i] = v
            assert L.sae_linear_ce_forward(C.byref(d), *args, 1 << 30, None) == sb.ERR_INVALID_ARG, (i, v)
    assert L.sae_linear_ce_forward(C.byref(withbias), *good, 1 << 30, None) == sb.ERR_INVALID_ARG
    assert L.sae_linear_ce_forward(None, *good, 1 << 30, None) == sb.ERR_INVALID_ARG
    good = [p, p, p, None, p, p, p, p, p, None, p]
    for i in (0, 1, 2, 4, 5, 6, 10):
        for v in (None, odd):
            args = list(good)
            args[i] = v
            assert L.sae_linear_ce_backward(C.byref(d), *args, 1 << 30, None) == sb.ERR_INVALID_ARG, (i, v)
    for i in (7, 8):
        args = list(good)
        args[i] = odd
        assert L.sae_linear_ce_backward(C.byref(d), *args, 1 << 30, None) == sb.ERR_INVALID_ARG
    args = list(good)
    args[9] = p                                             # a bias gradient without a bias
    assert L.sae_linear_ce_backward(C.byref(d), *args, 1 << 30, None) == sb.ERR_INVALID_ARG


def test_misaligned_rests_are_refused():
    L, p, odd = sb.lib(), C.c_void_p(256), C.c_void_p(257)
    d = desc()
    assert L.sae_linear_ce_forward_with_rest(C.byref(d), p, p, None, p, p, p, odd, p, p, 1 << 30, None) == sb.ERR_INVALID_ARG
    assert L.sae_linear_ce_backward_with_rest(C.byref(d), p, p, p, None, p, p, odd, p, p, p, None, p, 1 << 30, None) == sb.ERR_INVALID_ARG
    assert L.sae_linear_ce_backward_with_rest(C.byref(d), p, p, p, None, p, None, p, p, p, p, None, p, 1 << 30, None) == sb.ERR_INVALID_ARG


def test_module_arguments():
    with pytest.raises(ValueError):
        ce.LinearCrossEntropy(0, 3)
    with pytest.raises(ValueError):
        ce.LinearCrossEntropy(3, 3, reduction="max")
    m = ce.LinearCrossEntropy(6, 3)
    assert m.logits(torch.ones(2, 6)).shape == (2, 3) and ce.LinearCrossEntropy(6, 3, bias=False).bias is None


def test_host_tensors_are_refused():
    x, w, t = torch.ones(4, 8), torch.ones(5, 8), torch.zeros(4, dtype=torch.long)
    with pytest.raises(ValueError):
        ce.linear_cross_entropy_forward(x, w, t)
    with pytest.raises(ValueError):
        ce.linear_cross_entropy(x, w, t, reduction="max")


# ---- the definition ---------------------------------------------------------------------------------------------------------------

def data(n, d, v, dtype, bias=False, ignored=0.0, seed=0, scale=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, d), device="cuda", generator=gen).to(dtype)
    w = (torch.randn((v, d), device="cuda", generator=gen) * scale / math.sqrt(d)).to(dtype)
    b = (0.5 * torch.randn(v, device="cuda", generator=gen)).to(dtype) if bias else None
    t = torch.randint(v, (n,), device="cuda", generator=gen)
    t[torch.rand(n, device="cuda", generator=gen) < ignored] = IGNORE
    return x, w, t, b


class Exact:
    """Everything in float64, and how far a result may be off.

    u: half a step of the type.  dz: of a logit: every product of 16-bit values is exact in float; the sum of d terms loses at most one
    step 2^-23 of the sum of magnitudes for each 16 terms and for the joins (float32: parts leave out terms below 2^-23 of a product).
    The softmax adds the rounding of (z - m) log2(e) and of the exponential, 2^-22 (2 + |z|), and of the sums, 2^-24 for each
    term that a thread adds.  p is rounded to the type once, the results once."""

    def __init__(self, x, w, t, b, reduction, dloss=None):
        self.dtype, used = x.dtype, t != IGNORE
        x, w = x.double(), w.double()
        b = None if b is None else b.double()
        z = x @ w.t() + (0 if b is None else b)
        self.lse = torch.where(used, torch.logsumexp(z, 1), 0.0)
        rows = torch.where(used, self.lse - z.gather(1, torch.where(used, t, 0)[:, None])[:, 0], 0.0)
        self.count = int(used.sum())
        self.loss = {"none": rows, "sum": rows.sum(), "mean": rows.sum() / self.count if self.count else rows.sum() * math.nan}[reduction]
        n, d = x.shape
        v = len(w)
        mags = (x.abs() @ w.abs().t() + (0 if b is None else b.abs())).amax(1)
        self.dz = (d / 16 + 8) * 2.0 ** -23 * mags + 2.0 ** -22 * (2 + z.abs().amax(1)) + (v / 64 + 64) * 2.0 ** -24
        self.dloss_rows = 2 * self.dz
        self.loss_off = {"none": self.dloss_rows, "sum": self.dloss_rows[used].sum() + 2.0 ** -23 * rows.abs().sum(),
                         "mean": (self.dloss_rows[used].sum() + 2.0 ** -23 * rows.abs().sum()) / max(1, self.count)}[reduction]
        if dloss is None:
            return
        g = dloss.double() if reduction == "none" else dloss.double().expand(n) / (self.count if reduction == "mean" else 1)
        p = torch.exp(z - self.lse[:, None])
        both = p.clone()
        r = torch.arange(n, device="cuda")[used]
        p[r, t[used]] -= 1
        both[r, t[used]] += 1                            # what rounding before the subtraction is relative to
        g = torch.where(used, g, 0.0)[:, None]
        p, both = p * g, both * g.abs()
        u = 0.0 if self.dtype == torch.float32 else torch.finfo(self.dtype).eps / 2
        # a float16 p is scaled by 2^15 over the largest factor: half of its smallest step is 2^-25
        floor = 2.0 ** -40 * g.abs().max() if self.dtype == torch.float16 else 0.0
        dp = p.abs() * u + both * (2 * self.dz[:, None] + 2.0 ** -21) + floor
        dp = torch.where(used[:, None], dp, 0.0)
        end = torch.finfo(self.dtype).eps / 2
        tiny = torch.finfo(self.dtype).smallest_normal * torch.finfo(self.dtype).eps

        def off(result, s):
            return result.abs() * end + s * (1 + end) + tiny
        self.dx, self.dw, self.db = p @ w, p.t() @ x, p.sum(0)
        self.dx_off = off(self.dx, dp @ w.abs() + (v / 16 + 16) * 2.0 ** -23 * (p.abs() @ w.abs()))
        self.dw_off = off(self.dw, dp.t() @ x.abs() + (n / 16 + 16) * 2.0 ** -23 * (p.abs().t() @ x.abs()))
        self.db_off = off(self.db, dp.sum(0) + 40 * 2.0 ** -24 * p.abs().sum(0))


def near(got, want, off, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= off)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float(((got.double() - want).abs() / off).max())} of what is allowed"


def check(x, w, t, b, reduction, dloss):
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b, IGNORE, reduction)
    e = Exact(x, w, t, b, reduction, dloss)
    assert int(count) == e.count
    near(loss, e.loss, e.loss_off, "loss")
    near(lse, e.lse, torch.where(t != IGNORE, e.dloss_rows, 0.0), "lse")
    dx, dw, db = ce.linear_cross_entropy_backward(dloss, x, w, t, lse, count, b, IGNORE, reduction)
    assert dx.dtype == dw.dtype == x.dtype
    near(dx, e.dx, e.dx_off, "dx")
    near(dw, e.dw, e.dw_off, "dweight")
    if b is not None:
        off = e.db_off + e.db.abs() * (torch.finfo(b.dtype).eps / 2)
        near(db, e.db, off, "dbias")
    else:
        assert db is None


SIZES = [(1, 1, 1), (1, 8, 2), (2, 3, 5), (5, 64, 10), (31, 65, 63), (33, 40, 129), (127, 128, 64), (128, 64, 256), (129, 100, 257), (257, 77, 1000),
         (512, 192, 2049), (1000, 515, 333), (64, 2048, 1000), (16, 4096, 70), (3, 24, 20000), (2100, 16, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,v", SIZES)
def test_values_and_gradients(n, d, v, dtype):
    for i, (bias, ignored, reduction) in enumerate([(False, 0.0, "mean"), (True, 0.3, "none"), (True, 0.0, "sum")]):
        x, w, t, b = data(n, d, v, DTYPES[dtype], bias, ignored, seed=n + i)
        dloss = torch.rand(n, device="cuda") - 0.3 if reduction == "none" else torch.tensor(0.7, device="cuda")
        if int((t != IGNORE).sum()) == 0:
            t[0] = v - 1
        check(x, w, t, b, reduction, dloss)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,d,v,ignored", [("bf16", 4096, 256, 9000, 0.0), ("bf16", 20000, 64, 3000, 0.85), ("f16", 3000, 640, 7001, 0.1),
                                                 ("f32", 2000, 256, 3000, 0.2), ("bf16", 40000, 32, 300, 0.5), ("bf16", 9000, 128, 20000, 0.0),
                                                 ("bf16", 2500, 1100, 9000, 0.1), ("f16", 1500, 2048, 12000, 0.0), ("bf16", 16384, 96, 9000, 0.97)])
def test_large(dtype, n, d, v, ignored):
    """Pairs of blocks with one tile, several pieces of the classes, pieces wider for fewer rows, rows counted in two steps, sums long enough
    to be joined."""
    x, w, t, b = data(n, d, v, DTYPES[dtype], dtype != "bf16", ignored, seed=3)
    check(x, w, t, b, "mean", torch.tensor(1.0, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_factors_of_their_own_in_large_problems(dtype):
    """A dloss of its own for every row, of both signs and far apart, where tiles are shared by pairs of blocks."""
    x, w, t, b = data(3000, 512, 6001, DTYPES[dtype], True, 0.3, seed=21)
    dloss = torch.randn(3000, device="cuda") * 2.0 ** (torch.arange(3000, device="cuda") % 24 - 12)
    check(x, w, t, b, "none", dloss)


@pytest.mark.gpu
@pytest.mark.parametrize("ignored", [0.0, 0.3, 0.95])
def test_factors_of_their_own_for_rows_counted_in_two_steps(ignored):
    """float16 rows beyond what one block counts, each with its own dloss: three kernels in a chain before the first product, the last of which reads
    what the first has written.  Rows without a target in every run of 4096."""
    x, w, t, b = data(20000, 48, 300, torch.float16, True, ignored, seed=31)
    dloss = torch.randn(20000, device="cuda") * 2.0 ** (torch.arange(20000, device="cuda") % 16 - 8)
    for _ in range(3):
        check(x, w, t, b, "none", dloss)


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,v", [(256, 192, 64), (257, 192, 64), (256, 193, 64), (256, 192, 65), (255, 191, 63), (33, 20, 64), (32, 1, 1), (256, 512, 64), (255, 511, 63)])
def test_small_float_heads(n, d, v):
    """Where one launch takes them and just beyond: every reduction and type of bias, weights that start anywhere, an infinity, a masked
    class, a target that is none, nothing to count."""
    for i, reduction in enumerate(("mean", "sum", "none")):
        x, w, t, _ = data(n, d, v, torch.float32, False, 0.2, seed=n + i)
        t[0] = v - 1
        b = torch.randn(v, device="cuda").to(list(DTYPES.values())[i])
        dloss = torch.rand(n, device="cuda") - 0.3 if reduction == "none" else torch.tensor(0.7, device="cuda")
        check(x, w, t, b, reduction, dloss)
        want = ce.linear_cross_entropy_forward(x, w, t, b, reduction=reduction)
        flat = w.new_empty(w.numel() + 1)
        flat[1:] = w.reshape(-1)
        wide = x.new_full((n, d + 5), math.nan)
        wide[:, 3:3 + d] = x
        got = ce.linear_cross_entropy_forward(wide[:, 3:3 + d], flat[1:].view(v, d), t, b, reduction=reduction)
        assert all(torch.equal(p, q) for p, q in zip(want, got))
    rows = want[0]
    used = t != IGNORE
    bad = x.clone()
    bad[~used] = math.nan
    assert torch.equal(ce.linear_cross_entropy_forward(bad, w, t, b, reduction="none")[0], rows)
    others = torch.arange(n, device="cuda") != 0
    for value in (math.nan, math.inf):
        bad = x.clone()
        bad[0, d - 1] = value
        got = ce.linear_cross_entropy_forward(bad, w, t, b, reduction="none")[0]
        assert torch.equal(got[others], rows[others]) and torch.isnan(got[0])
    for value in (v, -1, 2 ** 40):
        wrong = t.clone()
        wrong[0] = value
        got = ce.linear_cross_entropy_forward(x, w, wrong, b, reduction="none")
        assert torch.equal(got[0][others], rows[others]) and torch.isnan(got[0][0]) and torch.equal(got[1], want[1])
        assert torch.isnan(ce.linear_cross_entropy_forward(x, w, wrong, b)[0])
    masked = b.float()
    masked[v - 1] = -math.inf
    got = ce.linear_cross_entropy_forward(x, w, t, masked, reduction="none")[0]
    assert float(got[0]) == math.inf if v > 1 else torch.isnan(got[0])
    if v > 1:
        keep = used & (t != v - 1)
        less = ce.linear_cross_entropy_forward(x, w[:-1], torch.where(keep, t, IGNORE), masked[:-1], reduction="none")[0]
        e = Exact(x, w[:-1], torch.where(keep, t, IGNORE), masked[:-1], "none")
        near(got[keep], e.loss[keep], e.loss_off[keep], "masked")
        near(less, e.loss, e.loss_off, "fewer classes")
    none = torch.full_like(t, IGNORE)
    assert float(ce.linear_cross_entropy_forward(x, w, none, b, reduction="sum")[0]) == 0 and torch.isnan(ce.linear_cross_entropy_forward(x, w, none, b)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("n,d,v", [(1, 40, 6000), (8, 64, 5001), (9, 61, 4099), (40, 132, 2049), (33, 1000, 2048)])
def test_few_float_rows(n, d, v):
    """A row's classes in several blocks, up to 8 rows in a tile and more; x that starts on no 16 bytes beside weights that do, and the
    other way round: the bits of the plain tensors."""
    for i, reduction in enumerate(("mean", "sum", "none")):
        x, w, t, b = data(n, d, v, torch.float32, i > 0, 0.2, seed=n + i)
        t[0] = v - 1
        dloss = torch.rand(n, device="cuda") - 0.3 if reduction == "none" else torch.tensor(0.7, device="cuda")
        check(x, w, t, b, reduction, dloss)
        want = ce.linear_cross_entropy_forward(x, w, t, b, reduction=reduction)
        grads = ce.linear_cross_entropy_backward(dloss, x, w, t, want[1], want[2], b, reduction=reduction)

        def off(a):
            return torch.cat([a.new_zeros((len(a), 3)), a], 1)[:, 3:]
        for xx, ww in ((off(x), w), (x, off(w))):
            got = ce.linear_cross_entropy_forward(xx, ww, t, b, reduction=reduction)
            again = ce.linear_cross_entropy_backward(dloss, xx, ww, t, got[1], got[2], b, reduction=reduction)
            assert all(torch.equal(p, q) for p, q in zip(want, got))
            assert all(p is q is None or torch.equal(p, q) for p, q in zip(grads, again))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(dtype):
    """Slices of wider tensors, odd offsets, an expanded row, transposed storage, more dimensions: the bits of the plain tensors."""
    x, w, t, b = data(96, 72, 200, DTYPES[dtype], True, 0.2, seed=5)
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b)
    one = torch.tensor(1.0, device="cuda")
    grads = ce.linear_cross_entropy_backward(one, x, w, t, lse, count, b)

    def wide(a, extra, at):
        big = a.new_full((a.shape[0], a.shape[1] + extra), math.nan)
        big[:, at:at + a.shape[1]] = a
        return big[:, at:at + a.shape[1]]

    def shifted(a):
        flat = a.new_empty(a.numel() + 1)
        flat[1:] = a.reshape(-1)
        return flat[1:].view(a.shape)
    for xx in (x, wide(x, 8, 0), wide(x, 37, 5), shifted(x), x.t().contiguous().t()):
        for ww in (w, wide(w, 16, 8), wide(w, 3, 1), shifted(w), w.t().contiguous().t()):
            got = ce.linear_cross_entropy_forward(xx, ww, t, b)
            assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
            again = ce.linear_cross_entropy_backward(one, xx, ww, t, got[1], got[2], b)
            assert all(torch.equal(p, q) for p, q in zip(grads, again))
    t2 = torch.stack([t, t], 1)[:, 0]
    assert torch.equal(ce.linear_cross_entropy_forward(x, w, t2, b)[0], loss)
    x3 = x.view(4, 24, 72)
    rows, lse3, count3 = ce.linear_cross_entropy_forward(x3, w, t.view(4, 24), b, reduction="none")
    assert rows.shape == lse3.shape == (4, 24)
    dx3 = ce.linear_cross_entropy_backward(torch.ones_like(rows), x3, w, t.view(4, 24), lse3, count3, b, reduction="none")[0]
    assert dx3.shape == x3.shape
    same = x[:1].expand(96, 72)
    assert torch.equal(ce.linear_cross_entropy_forward(same, w, t, b)[0], ce.linear_cross_entropy_forward(same.contiguous(), w, t, b)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_a_target_may_hold_anything(dtype):
    """NaN and infinities there reach nothing; the results are the bits of the remaining rows alone."""
    x, w, t, b = data(300, 40, 90, DTYPES[dtype], True, 0.5, seed=7)
    used = t != IGNORE
    one = torch.tensor(1.0, device="cuda")
    small = ce.linear_cross_entropy_forward(x[used], w, t[used], b)
    want = ce.linear_cross_entropy_backward(one, x[used], w, t[used], small[1], small[2], b)
    bad = x.clone()
    bad[~used] = torch.tensor([math.nan, math.inf, -math.inf, 1.0], device="cuda").to(x.dtype).repeat(10)
    loss, lse, count = ce.linear_cross_entropy_forward(bad, w, t, b)
    dx, dw, db = ce.linear_cross_entropy_backward(one, bad, w, t, lse, count, b)
    assert torch.equal(loss, small[0]) and torch.equal(lse[used], small[1]) and not lse[~used].any()
    assert torch.equal(dx[used], want[0]) and not dx[~used].any()
    assert torch.equal(dw, want[1]) and torch.equal(db, want[2])
    rows = ce.linear_cross_entropy_forward(bad, w, t, b, reduction="none")[0]
    assert not rows[~used].any()


@pytest.mark.gpu
def test_nothing_to_count():
    x, w, t, b = data(50, 16, 30, torch.bfloat16, True)
    t.fill_(IGNORE)
    one = torch.tensor(1.0, device="cuda")
    for reduction, want in (("mean", math.nan), ("sum", 0.0)):
        loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b, reduction=reduction)
        assert int(count) == 0 and (math.isnan(float(loss)) if math.isnan(want) else float(loss) == want)
        assert not any(g.any() for g in ce.linear_cross_entropy_backward(one, x, w, t, lse, count, b, reduction=reduction))
        empty = ce.linear_cross_entropy_forward(x[:0], w, t[:0], b, reduction=reduction)
        assert int(empty[2]) == 0 and (math.isnan(float(empty[0])) if math.isnan(want) else float(empty[0]) == want)
        dx, dw, db = ce.linear_cross_entropy_backward(one, x[:0], w, t[:0], empty[1], empty[2], b, reduction=reduction)
        assert dx.shape == (0, 16) and not dw.any() and not db.any()
    rows = ce.linear_cross_entropy_forward(x[:0], w, t[:0], b, reduction="none")
    assert rows[0].shape == (0,)
    dx, dw, db = ce.linear_cross_entropy_backward(rows[0], x[:0], w, t[:0], rows[1], rows[2], b, reduction="none")
    assert not dw.any() and not db.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_targets_that_are_none(dtype):
    """A target outside the classes makes its own loss and dx NaN and the sums over rows NaN; other rows stay."""
    x, w, t, b = data(40, 24, 17, DTYPES[dtype], False)
    want = ce.linear_cross_entropy_forward(x, w, t, reduction="none")[0]
    ones = torch.ones(40, device="cuda")
    good = ce.linear_cross_entropy_forward(x, w, t, reduction="none")
    dx0 = ce.linear_cross_entropy_backward(ones, x, w, t, good[1], good[2], reduction="none")[0]
    for value in (17, -1, 2 ** 40, -2 ** 40):
        bad = t.clone()
        bad[3] = value
        loss, lse, count = ce.linear_cross_entropy_forward(x, w, bad, reduction="none")
        others = torch.arange(40, device="cuda") != 3
        assert int(count) == 40 and torch.isnan(loss[3]) and torch.equal(loss[others], want[others])
        dx, dw, _ = ce.linear_cross_entropy_backward(ones, x, w, bad, lse, count, reduction="none")
        assert torch.isnan(dx[3]).all() and torch.equal(dx[others], dx0[others]) and torch.isnan(dw).all()
        assert torch.isnan(ce.linear_cross_entropy_forward(x, w, bad)[0])
    assert torch.equal(ce.linear_cross_entropy_forward(x, w, t, ignore_index=10 ** 12, reduction="none")[0], want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_classes_masked_by_the_bias(dtype):
    """A bias of -inf takes a class out: the others' results are those without it (whole tiles masked among them); a masked target's
    loss is infinite; a row that loses every class is NaN."""
    n, d, v = 70, 32, 700
    x, w, t, b = data(n, d, v, DTYPES[dtype], True, seed=2)
    keep = torch.ones(v, dtype=torch.bool, device="cuda")
    keep[64:400] = False
    keep[699] = False
    masked = b.clone()
    masked[~keep] = -math.inf
    names = keep.nonzero()[:, 0]
    t = names[t % len(names)]
    small_t = torch.cumsum(keep, 0)[t] - 1
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, masked, reduction="none")
    e = Exact(x, w[keep], small_t, b[keep], "none", torch.ones(n, device="cuda"))
    near(loss, e.loss, e.loss_off, "loss")
    dx, dw, db = ce.linear_cross_entropy_backward(torch.ones(n, device="cuda"), x, w, t, lse, count, masked, reduction="none")
    near(dx, e.dx, e.dx_off, "dx")
    near(dw[keep], e.dw, e.dw_off, "dweight")
    assert not dw[~keep].any() and not db[~keep].any()
    t[5] = 100
    assert float(ce.linear_cross_entropy_forward(x, w, t, masked, reduction="none")[0][5]) == math.inf
    masked.fill_(-math.inf)
    assert torch.isnan(ce.linear_cross_entropy_forward(x, w, t, masked, reduction="none")[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_stay_in_their_row(dtype, value):
    x, w, t, b = data(200, 24, 333, DTYPES[dtype], True, seed=4)
    want = ce.linear_cross_entropy_forward(x, w, t, b, reduction="none")[0]
    x[77, 5] = value
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b, reduction="none")
    others = torch.arange(200, device="cuda") != 77
    assert torch.equal(loss[others], want[others]) and torch.isnan(loss[77])
    dx = ce.linear_cross_entropy_backward(torch.ones(200, device="cuda"), x, w, t, lse, count, b, reduction="none")[0]
    assert torch.isfinite(dx[others]).all() and torch.isnan(dx[77]).any()


@pytest.mark.gpu
def test_logits_far_apart():
    """Differences of thousands: nothing overflows, the softmax is one of the largest logits alone; equal logits give log(classes).
    511 and 512 are the same in bfloat16 (8 bits: steps of 2 from 256 on, 511 to the even 512), so the largest is there twice."""
    v = 513
    w = torch.zeros((v, 8), device="cuda", dtype=torch.bfloat16)
    w[:, 0] = torch.arange(v, device="cuda").to(torch.bfloat16)
    x = torch.zeros((4, 8), device="cuda", dtype=torch.bfloat16)
    x[:, 0] = torch.tensor([64.0, -64.0, 0.0, 2.0 ** 100], device="cuda").to(torch.bfloat16)
    t = torch.tensor([512, 0, 7, 512], device="cuda")
    loss = ce.linear_cross_entropy_forward(x, w, t, reduction="none")[0]
    two = (2 + math.log(2)) * 2.0 ** -22
    assert float(w[511, 0]) == 512 and float(loss[1]) == 0
    assert abs(float(loss[0]) - math.log(2)) <= two and abs(float(loss[3]) - math.log(2)) <= two
    assert abs(float(loss[2]) - math.log(v)) <= (2 + math.log(v)) * 2.0 ** -22
    t = torch.tensor([0, 512, 7, 0], device="cuda")
    loss = ce.linear_cross_entropy_forward(x, w, t, reduction="none")[0]
    assert abs(float(loss[0]) - 64.0 * 512 - math.log(2)) <= 64.0 * 512 * 2.0 ** -22
    assert float(loss[1]) == 64.0 * 512 and float(loss[3]) == 512 * 2.0 ** 100


def gradients(x, w, t, b, reduction, dloss, how):
    """By the two calls, with lse as it came, or as a copy; and by autograd."""
    if how == "autograd":
        p = [None if a is None else a.clone().requires_grad_() for a in (x, w, b)]
        loss = ce.linear_cross_entropy(p[0], p[1], t, p[2], reduction=reduction)
        grads = torch.autograd.grad(loss, [a for a in p if a is not None], dloss)
        return tuple(grads) + (None,) * (3 - len(grads))
    _, lse, count = ce.linear_cross_entropy_forward(x, w, t, b, reduction=reduction)
    return ce.linear_cross_entropy_backward(dloss, x, w, t, lse.clone() if how == "copy" else lse, count, b, reduction=reduction)


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["calls", "autograd", "copy"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,v", [(1, 8, 50), (70, 20, 64), (300, 24, 1000), (600, 40, 3000)])
@pytest.mark.parametrize("offset", [256.0, 2992.0, 29952.0])
def test_gradients_at_large_logits(offset, n, d, v, dtype, how):
    """All logits of a row moved by the same number: the gradients are those without it, and so is what they may be off.  x and w are multiples
    of 1/4 and 1/8, offsets and their sums multiples of 1/32 below 2^15: every logit is exact in 20 bits.  Half of the rows have the largest logit's class
    for a target: there p - 1 is a small difference."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randint(-16, 17, (n, d), device="cuda", generator=gen).div(4).to(DTYPES[dtype])
    w = torch.randint(-16, 17, (v, d), device="cuda", generator=gen).div(8).to(DTYPES[dtype])
    b = torch.randint(-32, 33, (v,), device="cuda", generator=gen).div(32)
    x[:, 0], w[:, 0] = 1, offset
    t = torch.randint(v, (n,), device="cuda", generator=gen)
    t[::2] = (x[:, 1:].double() @ w[:, 1:].double().t() + b.double()).argmax(1)[::2]
    dloss = torch.rand(n, device="cuda", generator=gen) + 0.5
    e = Exact(x[:, 1:], w[:, 1:], t, b, "none", dloss)
    dx, dw, db = gradients(x, w, t, b, "none", dloss, how)
    near(dx[:, 1:], e.dx, e.dx_off, "dx")
    near(dw[:, 1:], e.dw, e.dw_off, "dweight")
    near(db, e.db, e.db_off + 2.0 ** -24 * e.db.abs(), "dbias")


@pytest.mark.gpu
def test_the_rest_of_lse():
    """What comes beside lse: a float's half step at most, their sum the exact value (log of a sum of 1000 terms within 2^-20, on exact logits); 0 where
    lse is; refused where it is none of this call's."""
    x, w, t, _ = data(100, 8, 1000, torch.bfloat16, False, 0.3)
    x, w = (x * 4).round() / 4, (w * 8).round() / 8
    x[:, 0], w[:, 0] = 1, 29952
    _, lse, count = ce.linear_cross_entropy_forward(x, w, t)
    want = torch.where(t != IGNORE, torch.logsumexp(x.double() @ w.double().t(), 1), 0.0)
    assert float((lse.double() + lse.rest.double() - want).abs().max()) <= 2.0 ** -20
    assert float(lse.rest.abs().max()) <= 2.0 ** -10 and not lse.rest[t == IGNORE].any()
    one = torch.ones((), device="cuda")
    whole = lse.rest
    for bad in (whole[:50], whole.double(), whole.cpu(), whole.repeat(2)[::2]):
        lse.rest = bad
        with pytest.raises(ValueError):
            ce.linear_cross_entropy_backward(one, x, w, t, lse, count)


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["calls", "autograd", "copy"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [3, 700])
def test_gradients_of_tied_classes(n, dtype, how):
    """Two classes at 2^25, 3998 at 0: p is 1/2 and 1/2 (half a step of the type and the few roundings of a softmax)."""
    x, w = torch.zeros((n, 16), device="cuda", dtype=DTYPES[dtype]), torch.zeros((4000, 16), device="cuda", dtype=DTYPES[dtype])
    x[:, 0], w[5, 0], w[3007, 0] = 4096, 8192, 8192
    w[5, 1], w[3007, 2] = 1, 1
    t = torch.full((n,), 5, device="cuda")
    dx = gradients(x, w, t, None, "sum", torch.tensor(1.0, device="cuda"), how)[0]
    want = torch.zeros_like(dx[0], dtype=torch.float64)
    want[1], want[2] = -0.5, 0.5
    assert float((dx.double() - want)[:, 1:].abs().max()) <= 2.0 ** -20


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["calls", "autograd", "copy"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d,v", [(1, 100, 60), (7, 192, 64), (256, 192, 64), (40, 700, 500), (300, 769, 900), (700, 1100, 2000), (2000, 2500, 700)])
def test_p_of_a_row_adds_up_to_nothing(n, d, v, dtype, how):
    """Logits of tens of thousands whose sums are not exact: the backward pass has to meet the logits that lse was made from, to the last bit.
    A feature that is 0 in x and 1 in every class has dx = the sum of a row's p, which is 0.  The softmax is one class (differences of thousands), so
    that is p of it and of the target, each off by half a step of the type and 2^-21 of its own, and the largest sum of exponentials by
    (v / 64 + 64) 2^-24."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((n, d), device="cuda", generator=gen).to(DTYPES[dtype])
    w = (torch.randn((v, d), device="cuda", generator=gen) * (20000 / math.sqrt(d))).to(DTYPES[dtype])
    x[:, d - 1], w[:, d - 1] = 0, 1
    t = torch.randint(v, (n,), device="cuda", generator=gen)
    t[::2] = (x.double() @ w.double().t()).argmax(1)[::2]
    dx = gradients(x, w, t, None, "none", torch.ones(n, device="cuda"), how)[0]
    u = 0.0 if dtype == "f32" else torch.finfo(DTYPES[dtype]).eps / 2
    assert float(dx[:, d - 1].abs().max()) <= 2 * (u + 2 * (2.0 ** -21 + (v / 64 + 64) * 2.0 ** -24))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long_sums_of_one_sign(dtype):
    """x and every p that is looked at are positive, so whatever the products cut off of their sums is of one sign, and shows in the mean over all elements of
    dweight, where the roundings of p and of the result (2^-11 or 2^-8, of both signs) leave 2^-8 / sqrt(127 * 4096), below 1e-5.  Sums are joined every 4096
    terms (float16) or 32768 at the latest: 256 or 2048 products of 16, each of which may cut off two steps, 2^-22, of a sum that grows evenly: 2^-23 for each."""
    n, d, v = 1 << 18, 4096, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = (torch.rand((n, d), device="cuda", generator=gen, dtype=torch.float16) + 0.5).to(DTYPES[dtype])
    w = torch.randn((v, d), device="cuda", generator=gen).mul_(0.3 / math.sqrt(d)).to(DTYPES[dtype])
    t = torch.zeros(n, device="cuda", dtype=torch.long)
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t)
    dw = ce.linear_cross_entropy_backward(torch.tensor(1000.0, device="cuda"), x, w, t, lse, count, need_x=False)[1]
    want = torch.zeros((v, d), device="cuda", dtype=torch.float64)
    for part in x.split(1 << 14):
        p = torch.softmax(part.double() @ w.double().t(), 1)
        p[:, 0] -= 1
        want += p.t() @ part.double()
    want *= 1000.0 / n
    off = ((dw.double() - want) / want)[1:].mean()
    assert abs(float(off)) <= (256 if dtype == "f16" else 2048) * 2.0 ** -23 + 1e-5, float(off)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [64, 1200])
def test_long_sums_over_the_classes(n):
    """The same of dx: weights between 1/2 and 3/2, the target's own part (its weights, exactly) taken out again."""
    d, v = 256, 1 << 19
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.rand((v, d), device="cuda", generator=gen, dtype=torch.float16) + 0.5
    x = torch.randn((n, d), device="cuda", generator=gen).mul_(0.02).half()
    t = torch.randint(v, (n,), device="cuda", generator=gen)
    w[t] = 0                                            # the target's p - 1 then adds nothing
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, reduction="sum")
    dx = ce.linear_cross_entropy_backward(torch.tensor(1.0, device="cuda"), x, w, t, lse, count, reduction="sum", need_weight=False)[0]
    top, total, want = (x.double() @ w.double().t()).amax(1, keepdim=True), 0.0, 0.0
    for part in w.split(1 << 16):
        q = torch.exp(x.double() @ part.double().t() - top)
        total, want = total + q.sum(1, keepdim=True), want + q @ part.double()
    off = ((dx.double() - want / total) / (want / total)).mean()
    assert abs(float(off)) <= 256 * 2.0 ** -23 + 1e-5, float(off)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("left", [0, 1, 300, 9000])
def test_few_rows_left_of_many(left, dtype):
    """Launches made for 9000 rows and 40000 classes, whose sums would be joined, where few rows take part, or none."""
    x, w, t, b = data(9000, 40, 40000, DTYPES[dtype], True, 0.0, seed=12)
    t[torch.randperm(9000, device="cuda")[left:]] = IGNORE
    if left:
        check(x, w, t, b, "mean", torch.tensor(1.0, device="cuda"))
    one = torch.tensor(1.0, device="cuda")
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b, reduction="sum")
    for some in (lse, lse.clone()):
        dx, dw, db = ce.linear_cross_entropy_backward(one, x, w, t, some, count, b, reduction="sum")
        assert int(count) == left and not dx[t == IGNORE].any() and torch.isfinite(dx).all() and torch.isfinite(dw).all()
        if not left:
            assert float(loss) == 0 and not dw.any() and not db.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,d,v", [("f32", 20, 64, 10), ("f32", 20, 300, 500), ("f32", 700, 64, 900), ("bf16", 700, 900, 3000), ("f16", 300, 65, 200)])
def test_the_entry_points_without_rest(dtype, n, d, v):
    """Loss and lse to the bit; the gradients those of a call with a copy of lse, and within the bounds of the ones with rest."""
    x, w, t, b = data(n, d, v, DTYPES[dtype], True, 0.2, seed=13)
    L, one = sb.lib(), torch.tensor(1.0, device="cuda")
    kind = {"f32": sb.TYPE_FLOAT, "bf16": sb.TYPE_BFLOAT, "f16": sb.TYPE_HALF}[dtype]
    s = desc(type=kind, bias_type=kind, has_bias=1, rows=n, features=d, classes=v, x_pitch=d, weight_pitch=d)
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b)
    want = ce.linear_cross_entropy_backward(one, x, w, t, lse.clone(), count, b)
    loss2, lse2, count2 = torch.full_like(loss, 7), torch.full_like(lse, 7), torch.full_like(count, 7)
    got = [torch.full_like(a, 7) for a in (x, w, b)]
    stream = torch.cuda.current_stream().cuda_stream
    need = [L.sae_linear_ce_workspace(C.byref(s), w.data_ptr(), k) for k in (0, 1)]
    ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")
    assert L.sae_linear_ce_forward(C.byref(s), x.data_ptr(), w.data_ptr(), b.data_ptr(), t.data_ptr(), loss2.data_ptr(), lse2.data_ptr(), count2.data_ptr(),
                                   ws.data_ptr(), need[0], stream) == sb.OK
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2) and torch.equal(count, count2)
    assert L.sae_linear_ce_backward(C.byref(s), one.data_ptr(), x.data_ptr(), w.data_ptr(), b.data_ptr(), t.data_ptr(), lse2.data_ptr(), count2.data_ptr(),
                                    got[0].data_ptr(), got[1].data_ptr(), got[2].data_ptr(), ws.data_ptr(), need[1], stream) == sb.OK
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    e = Exact(x, w, t, b, "mean", one)
    near(got[0], e.dx, e.dx_off, "dx")
    near(got[1], e.dw, e.dw_off, "dweight")
    near(got[2], e.db, e.db_off + e.db.abs() * (torch.finfo(b.dtype).eps / 2), "dbias")


@pytest.mark.gpu
def test_same_bits_again():
    for dtype, n in (("bf16", 3000), ("f32", 500)):
        x, w, t, b = data(n, 200, 5000, DTYPES[dtype], True, 0.1, seed=9)
        first = None
        for _ in range(3):
            out = ce.linear_cross_entropy_forward(x, w, t, b)
            out += ce.linear_cross_entropy_backward(torch.tensor(1.0, device="cuda"), x, w, t, out[1], out[2], b)
            first = first or out
            assert all(torch.equal(p, q) for p, q in zip(first, out))


@pytest.mark.gpu
def test_wanted_gradients_only():
    x, w, t, b = data(60, 40, 100, torch.bfloat16, True, 0.1)
    one = torch.tensor(1.0, device="cuda")
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b)
    whole = ce.linear_cross_entropy_backward(one, x, w, t, lse, count, b)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        got = ce.linear_cross_entropy_backward(one, x, w, t, lse, count, b, need_x=need[0], need_weight=need[1], need_bias=need[2])
        for g, f, n in zip(got, whole, need):
            assert (g is None) if not n else torch.equal(g, f)


# ---- autograd -------------------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_autograd_is_the_two_calls(reduction):
    x, w, t, b = data(90, 48, 120, torch.float32, True, 0.2)
    p = [v.clone().requires_grad_() for v in (x, w, b)]
    loss = ce.linear_cross_entropy(p[0], p[1], t, p[2], reduction=reduction)
    weights = torch.rand_like(loss)
    (loss * weights).sum().backward()
    fwd = ce.linear_cross_entropy_forward(x, w, t, b, reduction=reduction)
    want = ce.linear_cross_entropy_backward(weights, x, w, t, fwd[1], fwd[2], b, reduction=reduction)
    assert torch.equal(loss, fwd[0]) and all(torch.equal(a.grad, g) for a, g in zip(p, want))


@pytest.mark.gpu
def test_differences():
    """The gradient along a random direction against central differences of the float64 loss's own value as the kernel gives it: step h
    leaves h^2 / 6 of the third derivative (at most 2 |dz|^3 of the softmax) and the loss's own error over h."""
    x, w, t, b = data(40, 32, 60, torch.float32, True, 0.1, seed=11)
    one = torch.tensor(1.0, device="cuda")
    loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b)
    grads = ce.linear_cross_entropy_backward(one, x, w, t, lse, count, b)
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = 2.0 ** -6
    for i, base in enumerate((x, w, b)):
        direction = torch.randn(base.shape, device="cuda", generator=gen) * (0.1 if i < 2 else 1.0)
        values = []
        for sign in (1, -1):
            args = [x, w, b]
            args[i] = base + sign * h * direction
            values.append(float(ce.linear_cross_entropy_forward(args[0], args[1], t, args[2])[0]))
        slope = (values[0] - values[1]) / (2 * h)
        want = float((grads[i].double() * direction.double()).sum())
        moved = (direction @ w.t() if i == 0 else x @ direction.t() if i == 1 else direction.expand(40, 60)).abs().amax(1).double()
        e = Exact(x, w, t, b, "mean")
        allowed = float((h * h / 6 * 2 * (2 * moved) ** 3).mean()) + float(e.loss_off) / h + abs(want) * 1e-4
        assert abs(slope - want) <= allowed, (i, slope, want, allowed)


@pytest.mark.gpu
def test_module_under_autocast():
    torch.manual_seed(0)
    m = ce.LinearCrossEntropy(64, 50).cuda()
    x, t = torch.randn(30, 64, device="cuda"), torch.randint(50, (30,), device="cuda")
    with torch.autocast("cuda", torch.bfloat16):
        loss = m(x, t)
    loss.backward()
    assert m.weight.grad.dtype == torch.float32 and loss.dtype == torch.float32
    xb, wb = x.bfloat16(), m.weight.detach().bfloat16()
    fwd = ce.linear_cross_entropy_forward(xb, wb, t, m.bias.detach())
    want = ce.linear_cross_entropy_backward(torch.tensor(1.0, device="cuda"), xb, wb, t, fwd[1], fwd[2], m.bias.detach())
    assert torch.equal(loss, fwd[0]) and torch.equal(m.weight.grad, want[1].float()) and torch.equal(m.bias.grad, want[2])


@pytest.mark.gpu
def test_a_changed_input_is_noticed():
    x, w, t, _ = data(20, 16, 30, torch.float32)
    w.requires_grad_()
    loss = ce.linear_cross_entropy(x, w, t)
    with torch.no_grad():
        w.mul_(2)
    with pytest.raises(RuntimeError):
        loss.backward()


# ---- streams, graphs, devices ------------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
def test_on_another_stream_and_captured():
    x, w, t, b = data(700, 96, 3000, torch.bfloat16, True, 0.3, seed=6)
    one = torch.tensor(1.0, device="cuda")

    def both():
        loss, lse, count = ce.linear_cross_entropy_forward(x, w, t, b)
        return (loss,) + ce.linear_cross_entropy_backward(one, x, w, t, lse, count, b)
    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = both()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(both())
    x2, w2, t2, b2 = data(700, 96, 3000, torch.bfloat16, True, 0.6, seed=16)       # other rows take part
    for a, c in ((x, x2), (w, w2), (t, t2), (b, b2)):
        a.copy_(c)
    for g in graphs + graphs:
        g.replay()
    want = both()
    for out in outs:
        assert all(torch.equal(p, q) for p, q in zip(want, out))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,d,v", [("f32", 100, 64, 10), ("bf16", 300, 64, 500)])
def test_captured_training(dtype, n, d, v):
    """Loss and gradients by autograd inside a graph, replayed on other data; eager calls of other leaves go on beside it."""
    x, w, t, b = data(n, d, v, DTYPES[dtype], True, 0.2, seed=8)
    leaves = [a.clone().requires_grad_() for a in (x, w, b)]

    def both(p, t):
        loss = ce.linear_cross_entropy(p[0], p[1], t, p[2])
        return (loss.detach(),) + torch.autograd.grad(loss * 3, p)
    both(leaves, t)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both(leaves, t)
    x2, w2, t2, b2 = data(n, d, v, DTYPES[dtype], True, 0.5, seed=18)
    with torch.no_grad():
        for p, q in zip(leaves, (x2, w2, b2)):
            p.copy_(q)
    t.copy_(t2)
    want = both([a.clone().requires_grad_() for a in (x2, w2, b2)], t2)
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


@pytest.mark.gpu
def test_two_calls_at_once():
    a, c = data(2000, 128, 4000, torch.bfloat16, True, 0.1, seed=1), data(1500, 256, 3000, torch.bfloat16, False, 0.2, seed=2)
    want = [ce.linear_cross_entropy_forward(*d)[0] for d in (a, c)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, d in enumerate((a, c)):
            with torch.cuda.stream(streams[i]):
                got[i].append(ce.linear_cross_entropy_forward(*d)[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


@pytest.mark.gpu
def test_bad_calls_are_refused():
    x, w, t, b = data(8, 16, 10, torch.bfloat16, True)
    f = ce.linear_cross_entropy_forward
    for args in ((x.cpu(), w, t), (x, w.cpu(), t), (x, w, t.cpu()), (x.double(), w.double(), t), (x, w.float(), t), (x, w[:, :8], t), (x, w, t.int()), (x, w, t[:4]),
                 (x, w, t, b[:4]), (x, w, t, b.double()), (x, w, t, b.cpu()), (x, w, t, b.repeat(2)[::2]), (x, w[0], t), (x[:, :0], w[:, :0], t), (x, w[:0], t)):
        with pytest.raises(ValueError):
            f(*args)
    loss, lse, count = f(x, w, t, b)
    one = torch.ones((), device="cuda")
    g = ce.linear_cross_entropy_backward
    for args in ((one.double(), x, w, t, lse, count, b), (torch.ones(8, device="cuda"), x, w, t, lse, count, b), (one, x, w, t, lse[:4], count, b),
                 (one, x, w, t, lse.double(), count, b), (one, x, w, t, lse, count.float(), b), (one.cpu(), x, w, t, lse, count, b)):
        with pytest.raises(ValueError):
            g(*args)
    L = sb.lib()
    d = desc(rows=8, features=16, classes=10, x_pitch=16, weight_pitch=16)
    need = L.sae_linear_ce_workspace(C.byref(d), w.data_ptr(), 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    args = [x.data_ptr(), w.data_ptr(), None, t.data_ptr(), loss.data_ptr(), lse.data_ptr(), count.data_ptr(), ws.data_ptr()]
    assert need > 0 and L.sae_linear_ce_forward(C.byref(d), *args, need - 1, None) == sb.ERR_INVALID_ARG
