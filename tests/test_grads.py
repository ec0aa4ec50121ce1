"""Gradient sets (sae_grads_*): refusals, which need no GPU, and on the GPU norm, clip, pack and unpack against a plain
float64 computation.

Tolerances, with u = 2^-24: eight squares (or magnitudes) are summed in float, at most 8 roundings of positive terms,
then in double, so a sum is within 8u and its square root within 4u; rounding the norm to float adds u.  The scale
is taken from the double norm (8u for q = 1) and rounded (u); the product rounds once more: u to float32, 2^-8 to
bfloat16, 2^-11 to float16 (half a unit of the last place, relative), or half the smallest subnormal, absolute.  Clipping
in place rounds the scale to the tensor's type as well: once more the same."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2008_05823_b200 import binding as sb

U = 2.0 ** -24
SUM_TOL = {1: 8 * U, 2: 4 * U, math.inf: 0.0}
ROUND = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


# ---- refusals of the C entry points: nothing is launched --------------------------------------------------------------

def config(**kw):
    sizes = kw.pop("sizes", np.array([8, 8], dtype=np.int64))
    types = kw.pop("types", None)
    base = dict(abi_version=sb.ABI_VERSION, num_rows=2, num_tensors=len(sizes), device=0, stream=None,
                tensor_sizes=sizes.ctypes.data_as(C.POINTER(C.c_int64)),
                tensor_types=None if types is None else types.ctypes.data_as(C.POINTER(C.c_int32)))
    base.update(kw)
    cfg = sb.SaeGradsConfig(**base)
    cfg.held = (sizes, types)
    return cfg


@pytest.mark.parametrize("kw,status", [
    (dict(abi_version=7), sb.ERR_ABI), (dict(num_rows=0), sb.ERR_INVALID_ARG), (dict(num_rows=1025), sb.ERR_INVALID_ARG),
    (dict(num_tensors=0), sb.ERR_INVALID_ARG), (dict(tensor_sizes=None), sb.ERR_INVALID_ARG), (dict(device=-1), sb.ERR_INVALID_ARG),
    (dict(sizes=np.array([8, -1], dtype=np.int64)), sb.ERR_INVALID_ARG),
    (dict(sizes=np.array([8, 2 ** 30 + 1], dtype=np.int64)), sb.ERR_INVALID_ARG),
    (dict(types=np.array([0, 3], dtype=np.int32)), sb.ERR_INVALID_ARG)])
def test_init_refuses(kw, status):
    h = C.c_void_p(5)
    assert sb.lib().sae_grads_init(C.byref(config(**kw)), C.byref(h)) == status
    assert not h.value


def test_null_arguments_are_refused():
    L = sb.lib()
    fake = C.c_void_p(16)
    assert L.sae_grads_init(None, C.byref(C.c_void_p())) == sb.ERR_INVALID_ARG
    assert L.sae_grads_init(C.byref(config()), None) == sb.ERR_INVALID_ARG
    assert L.sae_grads_norm(None, fake, sb.NORM_TWO, fake) == sb.ERR_INVALID_ARG
    assert L.sae_grads_clip(None, fake, sb.NORM_TWO, 1.0, fake) == sb.ERR_INVALID_ARG
    assert L.sae_grads_pack(None, fake, sb.NORM_TWO, 1.0, fake, 0, fake) == sb.ERR_INVALID_ARG
    assert L.sae_grads_unpack(None, fake, 0, fake) == sb.ERR_INVALID_ARG
    L.sae_grads_destroy(None)


def test_init_without_a_device_fails_loudly():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    h = C.c_void_p()
    assert sb.lib().sae_grads_init(C.byref(config()), C.byref(h)) == sb.ERR_CUDA
    assert not h.value and sb.lib().sae_grads_last_cuda_error(None) != 0


# ---- the plain form -------------------------------------------------------------------------------------------------------

def flat64(row):
    return np.concatenate([t.detach().double().cpu().numpy().reshape(-1) for t in row] + [np.zeros(0)])


def norm64(v, q):
    if q == math.inf:
        return np.max(np.abs(v), initial=0.0)
    return math.sqrt(np.sum(v * v)) if q == 2 else np.sum(np.abs(v))


def coef64(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))


def assert_norms(got, rows, q):
    got = got.cpu().numpy().astype(np.float64)
    for k, row in enumerate(rows):
        want = norm64(flat64(row), q)
        assert abs(got[k] - want) <= (SUM_TOL[q] + U) * want, (k, got[k], want)


def assert_scaled(got, before, scale, dtype, q, in_place=False):
    """got ~ before * scale, rounded once to dtype; in place the scale is rounded to dtype too."""
    want = before * scale
    tol = np.abs(want) * (SUM_TOL[q] + 2 * U + (2 if in_place else 1) * ROUND[dtype]) + TINY[dtype]
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.flatnonzero(bad)[:5], got[bad][:5], want[bad][:5])


def make(K, sizes, dtypes, seed, offset=0):
    """K rows of tensors; `offset` elements into an allocation, so that nothing is aligned beyond the type."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = []
    for _ in range(K):
        row = []
        for j, (n, dt) in enumerate(zip(sizes, dtypes)):
            t = torch.randn(n + offset, device="cuda", generator=gen) * 10.0 ** (-(j % 4))
            row.append(t.to(dt)[offset:])
        rows.append(row)
    return rows


def gset(K, sizes, dtypes):
    from paper_2008_05823_b200 import grads
    return grads.GradSet(K, sizes, dtypes)


RAGGED = [1, 0, 7, 8, 9, 64, 8191, 8192, 8193, 3 * 8192 + 5, 2, 40000]
CASES = [
    (1, [1], [F32], 0), (1, [0], [F32], 0), (3, [0, 0], [F32, BF16], 0), (1, [8192], [BF16], 0), (2, [8193], [F16], 0),
    (1, RAGGED, [F32] * 12, 0), (3, RAGGED, [BF16] * 12, 0), (2, RAGGED, [F16] * 12, 0),
    (3, RAGGED, [F32, BF16, F16] * 4, 0), (3, RAGGED, [F32, BF16, F16] * 4, 1), (2, RAGGED, [BF16, F16, F32] * 4, 3),
    (2, RAGGED, [F32] * 12, 1), (2, RAGGED, [F32] * 12, 2), (1, [300000, 5], [F32, F32], 1),
    (5, [17, 100] * 30, [BF16, F32] * 30, 0),          # 300 pointers
    (9, [5, 33] * 50, [F32, BF16] * 50, 0),            # 900: through the pointer table
    (33, [3] * 130, [F32] * 130, 0),                   # 4290: more than one upload
    (1, [1000003, 12], [BF16, F32], 0), (40, [20011], [F32], 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("q", [1, 2, math.inf])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_norm_pack_clip_unpack(case, q):
    K, sizes, dtypes, offset = CASES[case]
    s = gset(K, sizes, dtypes)
    rows = make(K, sizes, dtypes, 10 + case, offset)
    assert_norms(s.norm(rows, q), rows, q)
    before = [flat64(r) for r in rows]
    norms = [norm64(v, q) for v in before]
    max_norm = float(np.float32(0.6 * max(norms) + 1e-3))        # some rows are scaled, some may not be
    # pack without a norm: the values themselves
    out, none = s.pack(rows)
    assert none is None
    assert np.array_equal(out.cpu().numpy().astype(np.float64), np.stack(before))
    # pack with clipping, into a wider buffer whose other columns stay
    wide = torch.full((K, s.d + 3), -7.0, device="cuda")
    out, got = s.pack(rows, wide[:, :s.d], max_norm=max_norm, norm_type=q)
    assert_norms(got, rows, q)
    for k in range(K):
        assert_scaled(wide[k, :s.d].double().cpu().numpy(), before[k], coef64(norms[k], max_norm), F32, q)
    assert bool((wide[:, s.d:] == -7.0).all())
    # the values back into tensors: rounded once
    back = make(K, sizes, dtypes, 99, offset)
    exact, _ = s.pack(rows)
    s.unpack(exact, back)
    for r, b in zip(rows, back):
        assert all(torch.equal(x, y) for x, y in zip(r, b))
    s.unpack(exact[K - 1], back)                                 # one vector for all
    for b in back:
        assert all(torch.equal(x, y) for x, y in zip(rows[K - 1], b))
    # in place
    got = s.clip_(rows, max_norm, q)
    for k in range(K):
        assert abs(float(got[k]) - norms[k]) <= (SUM_TOL[q] + U) * norms[k]
        at = 0
        for t, dt in zip(rows[k], dtypes):
            assert_scaled(t.double().cpu().numpy(), before[k][at:at + t.numel()], coef64(norms[k], max_norm), dt, q, in_place=True)
            at += t.numel()
    s.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("share", [0.3, 0.7, 0.9999, 1.5, 1e-7])
def test_clip_has_the_bits_of_a_product_in_place(dtype, share):
    """The tensors after clip_ are those of torch's in-place product with the float32 coefficient (here of the same norm)."""
    row = make(1, [7, 8192, 30011], [dtype] * 3, 8)[0]
    s = gset(1, [7, 8192, 30011], [dtype] * 3)
    norm = s.norm(row)
    max_norm = share * float(norm)
    want = [t.clone() for t in row]
    coef = (max_norm / (norm.double() + 1e-6)).clamp(max=1.0).float()[0]
    if share > 1e-6 or dtype != F16:                   # below a half's normal numbers the coefficient stays as it is
        for t in want:
            t.mul_(coef)
    else:
        want = [(t.float() * coef).half() for t in want]
    s.clip_(row, max_norm)
    near = torch.equal if dtype != F32 else (lambda a, b: torch.allclose(a, b, rtol=(4 + 3) * U, atol=0))
    assert all(near(a, b) for a, b in zip(row, want))


@pytest.mark.gpu
def test_unpack_rounds_to_nearest():
    v = torch.randn(5000, device="cuda")
    s = gset(1, [5000], [BF16])
    t = torch.empty(5000, device="cuda", dtype=BF16)
    s.unpack(v, [t])
    assert torch.equal(t, v.to(BF16))


@pytest.mark.gpu
def test_buffer_rows_and_row_strides():
    buf = torch.randn(6, 5001, device="cuda")
    s = gset(6, [5001], None)
    before = buf.double().cpu().numpy()
    norms = s.clip_(buf, 10.0)
    for k in range(6):
        want = norm64(before[k], 2)
        assert abs(float(norms[k]) - want) <= 5 * U * want
        assert_scaled(buf[k].double().cpu().numpy(), before[k], coef64(want, 10.0), F32, 2)
    wide = torch.randn(6, 6000, device="cuda")
    keep = wide[:, 5001:].clone()
    ref = gset(6, [5001], None).norm([[r.contiguous()] for r in wide[:, :5001]])
    assert torch.equal(s.norm(wide[:, :5001]), ref)
    s.clip_(wide[:, :5001], 1e-3)
    assert torch.equal(wide[:, 5001:], keep)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [1e30, 3e38, 1e-25, 1e-38, 1e-44, 0.0])
def test_range_of_the_squares(dtype, value):
    """Squares that overflow or vanish in float32 do not in the sum; float32 subnormals count."""
    n = 20000
    t = torch.full((n,), value, device="cuda", dtype=F32).to(dtype)
    s = gset(1, [n], [dtype])
    held = float(t[0].double())
    want = held * math.sqrt(n)
    got = float(s.norm([t])[0])
    if want > 3.4028235e38:
        assert got == math.inf
    else:
        assert abs(got - want) <= 5 * U * want + 2.0 ** -150
    mixed = t.clone()
    mixed[::97] = 1.0
    if value < 1:
        want = math.sqrt(norm64(flat64([mixed]), 2) ** 2)
        assert abs(float(s.norm([mixed])[0]) - want) <= 5 * U * want


@pytest.mark.gpu
@pytest.mark.parametrize("q", [1, 2, math.inf])
def test_infinities_and_nan(q):
    sizes = [9000, 100]
    rows = make(4, sizes, [F32, BF16], 3)
    rows[1][0][8200] = -math.inf
    rows[2][1][99] = math.nan
    rows[3][0][0], rows[3][1][5] = math.inf, math.nan
    clean = [t.clone() for t in rows[0]]
    s = gset(4, sizes, [F32, BF16])
    norms = s.norm(rows, q).cpu().numpy()
    assert np.isfinite(norms[0]) and norms[1] == np.inf and np.isnan(norms[2]) and np.isnan(norms[3])
    out, _ = s.pack(rows, max_norm=0.5, norm_type=q)
    out = out.cpu().numpy()
    assert np.isfinite(out[0]).all()
    assert np.isnan(out[1, 8200]) and not np.delete(out[1], 8200).any()
    assert np.isnan(out[2]).all() and np.isnan(out[3]).all()
    s.clip_(rows, math.inf, q)                                   # no limit: coef 1, but NaN where the norm is not finite
    assert all(torch.equal(a, b) for a, b in zip(clean, rows[0]))


@pytest.mark.gpu
def test_limits_of_max_norm():
    rows = make(2, [10000], [BF16], 4)
    keep = [r[0].clone() for r in rows]
    s = gset(2, [10000], [BF16])
    s.clip_(rows, 1e6)
    assert all(torch.equal(k, r[0]) for k, r in zip(keep, rows))
    s.clip_(rows, 0.0)
    assert all(not r[0].any() for r in rows)
    out, norms = s.pack(rows, max_norm=0.0)                      # norm 0: 0 / 1e-6
    assert not out.any() and not norms.any()


@pytest.mark.gpu
def test_same_bits_on_every_call_and_after_other_calls():
    rows = make(3, [100003, 77, 8192], [F32, BF16, F16], 5)
    s = gset(3, [100003, 77, 8192], [F32, BF16, F16])
    first, n1 = s.pack(rows, max_norm=1.0)
    first, n1 = first.clone(), n1.clone()
    for _ in range(20):
        s.norm(rows, 1)
        s.norm(rows, math.inf)
        out, n2 = s.pack(rows, max_norm=1.0)
        assert torch.equal(n1, n2) and torch.equal(out, first)


@pytest.mark.gpu
def test_channels_last_parameters_pack_in_memory_order():
    from paper_2008_05823_b200 import grads
    w = torch.randn(16, 3, 5, 5, device="cuda").to(memory_format=torch.channels_last)
    one = torch.randn(8, 4, 1, 1, device="cuda").to(memory_format=torch.channels_last)
    b = torch.randn(16, device="cuda")
    s = grads.GradSet.like([w, one, b])
    out, _ = s.pack([w, one, b])
    want = torch.cat([w.permute(0, 2, 3, 1).reshape(-1), one.reshape(-1), b])
    assert torch.equal(out[0], want)
    back = [torch.empty_like(w), torch.empty(8, 4, 1, 1, device="cuda"), torch.empty_like(b)]     # 1x1: either format
    s.unpack(out, back)
    assert torch.equal(back[0], w) and torch.equal(back[1], one) and torch.equal(back[2], b)
    with pytest.raises(ValueError):
        s.pack([w.contiguous(), one, b])


@pytest.mark.gpu
def test_rows_past_31_bits():
    """A row of more than 2^31 elements: the second half lands where it should."""
    n = 2 ** 30
    a = torch.zeros(n, device="cuda", dtype=BF16)
    b = torch.zeros(n, device="cuda", dtype=BF16)
    c = torch.arange(1, 1001, device="cuda", dtype=F32)
    a[-1], b[0], b[-1] = 2.0, 3.0, 4.0
    s = gset(1, [n, n, 1000], [BF16, BF16, F32])
    out, norms = s.pack([a, b, c], max_norm=1e9)
    assert [float(out[0, i]) for i in (n - 1, n, 2 * n - 1, 2 * n, 2 * n + 999)] == [2.0, 3.0, 4.0, 1.0, 1000.0]
    assert int(torch.count_nonzero(out)) == 1003
    want = math.sqrt(4 + 9 + 16 + sum(i * i for i in range(1, 1001)))
    assert abs(float(norms[0]) - want) <= 5 * U * want


@pytest.mark.gpu
def test_another_stream_and_graph_capture():
    sizes, dtypes = [50000, 333], [BF16, F32]
    rows = make(2, sizes, dtypes, 6)
    side = torch.cuda.Stream()
    s = gset(2, sizes, dtypes)
    want, wn = s.pack(rows, max_norm=1.0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                                # made on the default stream, called under another
        fresh = [[t * 1 for t in r] for r in rows]
        out, norms = s.pack(fresh, max_norm=1.0)
        total = out.sum(1)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(norms, wn) and torch.equal(total, want.sum(1))
    s.close()
    with torch.cuda.stream(side):
        s = gset(2, sizes, dtypes)
        out = torch.empty(2, s.d, device="cuda")
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            _, norms = s.pack(rows, out, max_norm=1.0)
        for r in rows:
            for t in r:
                t.mul_(2)
        g.replay()
        side.synchronize()
    assert torch.allclose(norms, 2 * wn, rtol=2 * U, atol=0) and torch.allclose(out, want, rtol=1e-5, atol=0)


@pytest.mark.gpu
def test_python_refusals():
    from paper_2008_05823_b200 import grads
    ok = make(2, [10, 20], [F32, BF16], 7)
    s = gset(2, [10, 20], [F32, BF16])
    a, b = ok[0]
    for bad in ([ok[0]], ok[0], [ok[0], [a]], [[a, b.float()], ok[1]], [[a.cpu(), b], ok[1]], [[a[:9], b], ok[1]],
                [[a, torch.zeros(40, device="cuda", dtype=BF16)[::2]], ok[1]], [[a, b[:1].expand(20)], ok[1]], []):
        with pytest.raises((ValueError, TypeError)):
            s.norm(bad)
    for out in (torch.empty(2, 31, device="cuda"), torch.empty(30, device="cuda"), torch.empty(2, 30),
                torch.empty(2, 30, device="cuda", dtype=BF16), torch.empty(30, 2, device="cuda").t(), torch.empty(1, 30, device="cuda").expand(2, 30)):
        with pytest.raises(ValueError):
            s.pack(ok, out)
    with pytest.raises(ValueError):
        s.norm(ok, norm_type=3)
    for bad in (-1.0, math.nan):
        with pytest.raises(sb.SaeError):
            s.clip_(ok, bad)
        with pytest.raises(sb.SaeError):
            s.pack(ok, max_norm=bad)
    with pytest.raises(ValueError):
        grads.GradSet(1, [4], torch.float64)
    with pytest.raises(ValueError):
        grads.GradSet(1, [4], device="cpu")
    with pytest.raises(sb.SaeError):
        grads.GradSet(0, [4])
    with pytest.raises(ValueError):
        grads.GradSet.like([torch.zeros(4, 4, device="cuda")[:, :2]])


@pytest.mark.gpu
def test_tensors_that_only_a_generator_holds():
    """The tensors of a generator live until the kernels that read them are enqueued: the call's own outputs are not in their place."""
    sizes, dtypes = [1, 90, 3, 128, 7], [F32, BF16, F32, F32, F16]
    rows = make(6, sizes, dtypes, 41)
    s, one = gset(6, sizes, dtypes), gset(1, sizes, dtypes)
    want, (out, _) = s.norm(rows), s.pack(rows, max_norm=0.5)
    for _ in range(20):
        assert torch.equal(s.norm((t * 1 for t in row) for row in rows), want)
        got, norms = s.pack(((t * 1 for t in row) for row in rows), max_norm=0.5)
        assert torch.equal(got, out) and torch.equal(norms, want)
        assert torch.equal(one.norm(t * 1 for t in rows[2]), want[2:3])


@pytest.mark.gpu
def test_autograd_sees_what_is_written():
    """unpack, clip_ and pack's out change tensors in place: a backward pass that needs what was there before raises, as it does
    after torch's own in-place operations; what is only read counts as unchanged."""
    s = gset(1, [12, 4], [F32, F32])
    vec = torch.randn(16, device="cuda")

    def forward():
        w = torch.randn(12, device="cuda", requires_grad=True)
        return w, torch.randn(4, device="cuda"), (w * w).sum()

    w, b, loss = forward()
    s.norm([w.detach(), b])
    s.pack([w, b])
    loss.backward()
    assert torch.equal(w.grad, 2 * w.detach())
    for write in (lambda w, b: s.unpack(vec, [w.detach(), b]), lambda w, b: s.clip_([w.detach(), b], 1e-3), lambda w, b: s.unpack(vec, [w, b])):
        w, b, loss = forward()
        before = w._version, b._version
        write(w, b)
        assert w._version > before[0] and b._version > before[1]
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    leaf = torch.ones(16, device="cuda", requires_grad=True)
    out = torch.ones(16, device="cuda")
    loss = (leaf * out).sum()
    s.pack([w.detach(), b], out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    buf = torch.ones(3, 5, device="cuda")
    gset(3, [5], None).clip_(buf, 0.1)
    assert buf._version == 1
    with torch.inference_mode():
        t = torch.ones(12, device="cuda"), torch.ones(4, device="cuda")
        s.unpack(vec, t)
    assert torch.equal(torch.cat(t), vec)


@pytest.mark.gpu
@pytest.mark.parametrize("q", [1, 2, math.inf])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_same_bits_at_every_alignment(dtype, q):
    """Equal values have equal norms wherever they lie: eight are added in float and the rest in double, in one order."""
    sizes = [5, 30011, 8192, 4099]
    s = gset(1, sizes, [dtype] * 4)
    row = make(1, sizes, [dtype] * 4, 12)[0]
    want = s.norm(row, q)
    out, _ = s.pack(row, max_norm=0.25, norm_type=q)
    for offset in range(1, 9):
        moved = [torch.cat([t[:offset], t])[min(offset, t.numel()):] for t in row]
        assert torch.equal(s.norm(moved, q), want), offset
        assert torch.equal(s.pack(moved, max_norm=0.25, norm_type=q)[0], out)
    # the rows of a buffer whose length is odd against 16 bytes
    one = torch.randn(16411, device="cuda").to(dtype)
    norms = gset(9, [16411], dtype).norm(one.repeat(9, 1), q)
    assert torch.equal(norms, norms[:1].expand(9))


@pytest.mark.gpu
def test_a_norm_beyond_float_still_scales():
    """Finite rows whose norm passes the largest float: it is reported as infinity, and the coefficient is right all the same."""
    n = 20000
    row = [torch.full((n,), 3e38, device="cuda"), torch.full((9,), -1e30, device="cuda")]
    s = gset(1, [n, 9], None)
    flat = flat64(row)
    out, norms = s.pack(row, max_norm=1e38)
    assert float(norms[0]) == math.inf
    assert_scaled(out[0].double().cpu().numpy(), flat, coef64(norm64(flat, 2), 1e38), F32, 2)


@pytest.mark.parametrize("shape", [(0,), (4, 0), (0, 4), (3, 0, 5)])
def test_a_tensor_of_nothing_has_no_gaps(shape):
    from paper_2008_05823_b200 import grads
    assert grads._fills_its_span(torch.empty(shape)) and grads._fills_its_span(torch.empty(shape).t() if len(shape) == 2 else torch.empty(shape))


@pytest.mark.gpu
def test_a_set_like_empty_tensors():
    from paper_2008_05823_b200 import grads
    w = torch.randn(3, 4, device="cuda")
    s = grads.GradSet.like([torch.empty(4, 0, device="cuda"), w, torch.empty(2, 0, 3, device="cuda")])
    out, _ = s.pack([torch.empty(0, 4, device="cuda").t(), w, torch.empty(2, 0, 3, device="cuda")])
    assert torch.equal(out[0], w.reshape(-1))


@pytest.mark.gpu
def test_a_closed_set_refuses():
    row = make(1, [8], [F32], 1)[0]
    s = gset(1, [8], None)
    s.close()
    s.close()
    for call in (lambda: s.norm(row), lambda: s.clip_(row, 1.0), lambda: s.pack(row), lambda: s.unpack(torch.zeros(8, device="cuda"), row)):
        with pytest.raises(sb.SaeError):
            call()
