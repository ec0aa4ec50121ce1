"""Orthogonalisation against its definition in float64: shapes, types, pitches, rows of workers, special values, streams, graphs,
refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2008_05823_b200 import binding as sb
from paper_2008_05823_b200 import orthogonal
from paper_2008_05823_b200.cross_entropy import linear_cross_entropy_forward
from paper_2008_05823_b200.orthogonal import COEFFICIENTS, Orthogonalizer

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


# ---- refusals, without a GPU ----------------------------------------------------------------------------------------------------

def init(rows=(4,), cols=(5,), types=None, results=None, steps=1, coefs=COEFFICIENTS, **kw):
    keep = [np.array(rows, dtype=np.int64), np.array(cols, dtype=np.int64), np.array(coefs * max(1, steps), dtype=np.float32)]
    i64, i32, f32 = (C.POINTER(t) for t in (C.c_int64, C.c_int32, C.c_float))
    arrays = [np.array(t, dtype=np.int32) if t is not None else None for t in (types, results)]
    base = dict(abi_version=sb.ABI_VERSION, num_rows=1, num_matrices=len(rows), rows=keep[0].ctypes.data_as(i64), cols=keep[1].ctypes.data_as(i64),
                types=arrays[0].ctypes.data_as(i32) if types is not None else None,
                result_types=arrays[1].ctypes.data_as(i32) if results is not None else None, steps=steps,
                coefficients=keep[2].ctypes.data_as(f32), eps=1e-7, device=0, stream=None)
    h = C.c_void_p()
    rc = sb.lib().sae_ortho_init(C.byref(sb.SaeOrthoConfig(**(base | kw))), C.byref(h))
    assert not h.value
    return rc


@pytest.mark.parametrize("bad", [dict(rows=(-1,)), dict(rows=((1 << 20) + 1,)), dict(rows=(1 << 20,), cols=(1 << 20,)), dict(types=(3,)), dict(results=(-1,)),
                                 dict(steps=0), dict(steps=65), dict(coefs=(math.nan, 0.0, 0.0)), dict(coefs=(40.0, 0.0, 0.0)), dict(coefs=(1.0, 0.0, 9000.0)),
                                 dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(num_rows=0), dict(num_rows=2000), dict(num_matrices=0),
                                 dict(device=-1)])
def test_bad_configurations_are_refused(bad):
    assert init(**bad) == sb.ERR_INVALID_ARG


def test_abi_and_null():
    L = sb.lib()
    assert init(abi_version=99) == sb.ERR_ABI
    assert L.sae_ortho_init(None, C.byref(C.c_void_p())) == sb.ERR_INVALID_ARG
    assert L.sae_ortho_run(None, None, None, None, None) == sb.ERR_INVALID_ARG
    assert L.sae_ortho_last_cuda_error(None) >= 0
    L.sae_ortho_destroy(None)


def test_python_arguments():
    for kw in (dict(shapes=[]), dict(shapes=[(4,)]), dict(shapes=[(4, 4)], dtypes=torch.float64), dict(shapes=[(4, 4)], dtypes=[torch.float32] * 2),
               dict(shapes=[(4, 4)], steps=0), dict(shapes=[(4, 4)], coefficients=(1.0, 2.0)), dict(shapes=[(4, 4)], steps=2, coefficients=[COEFFICIENTS] * 3),
               dict(shapes=[(4, 4)], device="cpu"), dict(shapes=[(4, 4)], result_dtypes=torch.int8)):
        with pytest.raises(ValueError):
            Orthogonalizer(**kw)
    with pytest.raises(ValueError):
        Orthogonalizer.like([])


# ---- the definition -----------------------------------------------------------------------------------------------------------------

def triples(steps, coefs):
    return [coefs] * steps if isinstance(coefs[0], float) else list(coefs)


def exact(g, steps=5, coefs=COEFFICIENTS, eps=1e-7):
    x = g.double().reshape(g.shape[0], -1)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for a, b, c in triples(steps, coefs):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return (x.t() if tall else x).reshape(g.shape)


def rounded(g, parts, steps=5, coefs=COEFFICIENTS, eps=1e-7):
    """The same in float64 with the documented roundings: x held as two float16 parts, products over `parts` of them."""
    def split(t, scale):
        hi = (t * scale).half().double()
        return [hi / scale, (t * scale - hi).half().double() / scale]

    def product(p, q):
        return sum(p[i] @ q[j] for i in range(parts) for j in range(parts) if i + j < parts)
    x = g.double().reshape(g.shape[0], -1)
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for a, b, c in triples(steps, coefs):
        xp = split(x, 2.0 ** 13)
        sp = split(product(xp, [v.t() for v in xp]), 2.0 ** 13)
        bp = split(b * sum(sp[:parts]) + c * product(sp, [v.t() for v in sp]), 2.0 ** 11)
        x = a * (xp[0] + xp[1]) + product(bp, xp)
    return (x.t() if tall else x).reshape(g.shape)


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


def gradient(shape, dtype, seed=0, kind="shared"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    m, n = shape[0], math.prod(shape[1:])
    g = torch.randn((m, n), device="cuda", generator=gen)
    if kind == "shared":                     # a few strong directions over noise
        r = min(4, m, n)
        g = 0.05 * g + torch.randn((m, r), device="cuda", generator=gen) @ torch.randn((r, n), device="cuda", generator=gen)
    return (g * 1e-3).reshape(shape).to(dtype)


def allowed(g, dtype):
    """Twice the error of the documented roundings, which the kernels make at other sums; the result's own rounding; and for the sums
    in float, which lose up to 2^-23 at each of 4 products of 16 before they are joined, three times a step: what 5 steps
    make of 36 2^-24, 3.4445^5 = 485 at most in the direction where it grows fastest and about 20 over a whole matrix."""
    one = dtype == torch.bfloat16 and min(g.shape[0], g[0].numel()) > 128
    return 2 * rel(rounded(g, 1 if one else 2), exact(g)) + torch.finfo(dtype).eps / 2 + 20 * 36 * 2.0 ** -24


SHAPES = [(1, 1), (1, 9), (7, 1), (2, 2), (16, 27), (64, 63), (65, 64), (100, 333), (333, 100), (128, 129), (129, 128), (200, 200), (257, 511), (600, 130),
          (131, 1100), (512, 768), (1000, 1001)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["noise", "shared"])
@pytest.mark.parametrize("dtype,result", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("bf16", "f32")])
def test_shapes_and_types(dtype, result, kind):
    gs = [gradient(s, DTYPES[dtype], i, kind) for i, s in enumerate(SHAPES)]
    plan = Orthogonalizer(SHAPES, DTYPES[dtype], result_dtypes=DTYPES[result])
    for g, y in zip(gs, plan(gs)):
        assert y.shape == g.shape and y.dtype == DTYPES[result]
        assert rel(y, exact(g)) <= allowed(g, DTYPES[result]), tuple(g.shape)


@pytest.mark.gpu
@pytest.mark.parametrize("result", ["bf16", "f32"])
def test_large_batches(result):
    """More tiles than there are clusters of blocks, tall, wide and square ones in one list, two rows of workers."""
    shapes = [(768, 768)] * 5 + [(1536, 700)] * 3 + [(700, 1536)] * 3 + [(2000, 300)] * 2
    rows = [[gradient(s, torch.bfloat16, 100 * k + i) for i, s in enumerate(shapes)] for k in range(2)]
    plan = Orthogonalizer(shapes, torch.bfloat16, num_rows=2, result_dtypes=DTYPES[result])
    out = plan(rows)
    for row, ys in zip(rows, out):
        for g, y in zip(row, ys):
            assert rel(y, exact(g)) <= allowed(g, DTYPES[result]), tuple(g.shape)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,result", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_long_sums(dtype, result):
    """Matrices whose square products are few and long are made in parts: wide, tall, odd, beside others that are not; the same bits again."""
    shapes = [(25, 3770), (3001, 140), (168, 2518), (129, 1001), (333, 1001), (200, 200), (300, 9000), (70, 50)]
    for group in ([s] for s in shapes), [shapes[:3] + shapes[5:]], [shapes]:
        for some in group:
            gs = [gradient(s, DTYPES[dtype], i) for i, s in enumerate(some)]
            plan = Orthogonalizer(some, DTYPES[dtype], result_dtypes=DTYPES[result])
            out = plan(gs)
            for g, x in zip(gs, out):
                assert rel(x, exact(g)) <= allowed(g, DTYPES[result]), tuple(g.shape)
            assert all(torch.equal(a, b) for _ in range(3) for a, b in zip(out, plan(gs)))


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2, 7])
def test_steps_and_coefficients(steps):
    g = gradient((150, 210), torch.float32, 3, "noise")
    for coefs in (COEFFICIENTS, (1.5, -0.5, 0.0), (2.0, -1.5, 0.5)):
        y = Orthogonalizer([g.shape], steps=steps, coefficients=coefs)([g])[0]
        assert rel(y, exact(g, steps, coefs)) <= 2 * rel(rounded(g, 2, steps, coefs), exact(g, steps, coefs)) + 2.0 ** -24 + 20 * 36 * 2.0 ** -24
    each = [(3.0, -3.0, 1.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)]
    y = Orthogonalizer([g.shape], steps=3, coefficients=each)([g])[0]
    assert rel(y, exact(g, 3, each)) <= 2 * rel(rounded(g, 2, 3, each), exact(g, 3, each)) + 20 * 37 * 2.0 ** -24


@pytest.mark.gpu
def test_singular_vectors_stay():
    """The result times the singular vectors is diagonal, and where the iteration has converged the values are near 1."""
    g = gradient((60, 90), torch.float32, 5, "noise")
    y = Orthogonalizer([g.shape], steps=20, coefficients=(1.875, -1.25, 0.375))([g])[0].double()
    u, _, vt = torch.linalg.svd(g.double(), full_matrices=False)
    assert float((y - u @ vt).norm()) <= 1e-4 * 60 ** 0.5
    assert float((y @ y.t() - torch.eye(60, device="cuda", dtype=torch.float64)).abs().max()) <= 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(dtype):
    """Pitches, odd offsets, channels-last convolutions, results with gaps: the bits of the plain tensors; what lies around stays."""
    dt = DTYPES[dtype]
    g = gradient((48, 75), dt, 1)
    plan = Orthogonalizer([(48, 75)], dt)
    want = plan([g])[0]

    def wide(a, extra, at):
        big = torch.full((a.shape[0], a.shape[1] + extra), 7.0, device="cuda", dtype=a.dtype)
        big[:, at:at + a.shape[1]] = a
        return big, big[:, at:at + a.shape[1]]

    flat = torch.full((g.numel() + 2,), 7.0, device="cuda", dtype=dt)
    flat[1:-1] = g.reshape(-1)
    for src in (g, wide(g, 5, 0)[1], wide(g, 53, 16)[1], flat[1:-1].view(48, 75)):
        big, dst = wide(torch.zeros_like(g), 21, 3)
        assert plan([src], [dst])[0] is dst and torch.equal(dst, want)
        assert (big[:, :3] == 7).all() and (big[:, 78:] == 7).all()
    inplace = flat[1:-1].view(48, 75)
    plan([inplace], [inplace])
    assert torch.equal(inplace, want) and float(flat[0]) == 7 and float(flat[-1]) == 7
    conv = gradient((32, 10, 3, 3), dt, 2)
    last = conv.contiguous(memory_format=torch.channels_last)
    p4 = Orthogonalizer.like([conv])
    a, b = p4([conv])[0], p4([last])[0]
    assert b.stride() == last.stride() and rel(a, exact(conv)) <= allowed(conv, dt) and rel(b, exact(conv)) <= allowed(conv, dt)
    with pytest.raises(ValueError):
        p4([conv], [torch.empty_like(last)])


@pytest.mark.gpu
def test_lists_and_mixed_types():
    shapes = [(40, 50), (300, 140), (0, 5), (40, 50), (6, 0), (140, 300), (3, 1000)]
    kinds = [torch.float32, torch.bfloat16, torch.float32, torch.float16, torch.bfloat16, torch.float32, torch.float16]
    results = [torch.bfloat16, torch.bfloat16, torch.float32, torch.float32, torch.bfloat16, torch.float16, torch.float16]
    plan = Orthogonalizer(shapes, kinds, num_rows=3, result_dtypes=results)
    rows = [[gradient(s, k, 10 * r + i) if 0 not in s else torch.zeros(s, dtype=k, device="cuda") for i, (s, k) in enumerate(zip(shapes, kinds))] for r in range(3)]
    out = plan(rows)
    again = plan((iter_row for iter_row in [tuple(r) for r in rows]))
    for row, ys, zs in zip(rows, out, again):
        for g, y, z, k in zip(row, ys, zs, results):
            assert y.shape == g.shape and y.dtype == k and torch.equal(y, z)
            if g.numel():
                assert rel(y, exact(g)) <= allowed(g, k)
    one = Orthogonalizer(shapes[:2], kinds[:2])
    assert isinstance(one([rows[0][0], rows[0][1]])[0], torch.Tensor) and isinstance(one([[rows[0][0], rows[0][1]]])[0], list)


@pytest.mark.gpu
def test_more_matrices_than_travel_as_arguments():
    shapes = [(8, 12)] * 500 + [(20, 9)] * 30
    gs = [gradient(s, torch.float32, i, "noise") for i, s in enumerate(shapes)]
    for g, y in zip(gs, Orthogonalizer(shapes)(gs)):
        assert rel(y, exact(g)) <= allowed(g, torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_shapes_and_batches_than_shared_memory_holds(dtype):
    """40 shapes and 7 steps, 840 products: both tables are read from memory.  33 shapes and 3 steps: one of them is."""
    kind = DTYPES[dtype]
    for count, steps in ((40, 7), (33, 3), (40, 6), (12, 23)):
        shapes = [(131 + 5 * i, 420 - 7 * i) if i % 2 else (300 - 3 * i, 140 + 9 * i) for i in range(count)]
        gs = [gradient(s, kind, i, "noise") for i, s in enumerate(shapes)]
        coefs = [(1.875, -1.25, 0.375)] * steps
        for g, y in zip(gs, Orthogonalizer(shapes, kind, steps=steps, coefficients=coefs)(gs)):
            one = 1 if kind == torch.bfloat16 else 2
            off = 2 * rel(rounded(g, one, steps, coefs), exact(g, steps, coefs)) + torch.finfo(kind).eps / 2 + 20 * 36 * 2.0 ** -24
            assert rel(y, exact(g, steps, coefs)) <= off, (count, steps, tuple(g.shape))


@pytest.mark.gpu
def test_many_small_and_large_matrices_in_one_list():
    """More than travel as arguments, of every kind: held by one SM or made tile by tile, in one part or two, their addresses in two tables."""
    small, large = [(8, 12), (64, 70), (100, 40), (128, 300)], [(200, 300), (131, 1100), (333, 140)]
    shapes = [large[i // 40 % 3] if i % 40 == 7 else small[i % 4] for i in range(470)]
    kinds = [(torch.float32, torch.bfloat16, torch.float16)[i % 3] for i in range(470)]
    results = [(torch.bfloat16, torch.float32)[i // 47 % 2] for i in range(470)]
    gs = [gradient(s, k, i) for i, (s, k) in enumerate(zip(shapes, kinds))]
    plan = Orthogonalizer(shapes, kinds, result_dtypes=results)
    out = plan(gs)
    for i, (g, y, k) in enumerate(zip(gs, out, results)):
        assert rel(y, exact(g)) <= allowed(g, k), (i, tuple(g.shape))
    assert all(torch.equal(a, b) for a, b in zip(out, plan(gs)))


@pytest.mark.gpu
@pytest.mark.parametrize("result", ["bf16", "f32"])
def test_lists_of_several_portions(result):
    """About 1.2 GB of workspace, gone through in portions of half a GB: shapes that begin in one and end in the next, whose S is made in parts or not."""
    shapes = [(2048, 1900)] * 14 + [(140, 9000)] * 6 + [(1000, 3000)] * 14
    gs = [gradient(s, torch.bfloat16, i) for i, s in enumerate(shapes)]
    plan = Orthogonalizer(shapes, torch.bfloat16, result_dtypes=DTYPES[result])
    out = plan(gs)
    for i, (g, y) in enumerate(zip(gs, out)):
        assert rel(y, exact(g)) <= allowed(g, DTYPES[result]), (i, tuple(g.shape))
    assert all(torch.equal(a, b) for a, b in zip(out, plan(gs)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_scales_and_special_values(dtype):
    """Norms from the smallest to the largest that the type holds; zeros; a matrix that is not finite is NaN and its neighbours stay."""
    dt = DTYPES[dtype]
    base = gradient((30, 40), torch.float32, 4, "noise") * 1e3
    top, low = (1e3, 1e-2) if dt == torch.float16 else (1e37, 1e-30)
    gs = [(base * top).to(dt), (base * low).to(dt), torch.zeros((30, 40), device="cuda", dtype=dt), base.to(dt), base.to(dt).clone(), base.to(dt).clone(), base.to(dt).clone()]
    gs[4][3, 7] = math.nan
    gs[5][29, 39] = math.inf
    gs[6][0, 0] = -math.inf
    plan = Orthogonalizer([(30, 40)] * 7, dt, eps=1e-7)
    y = plan(gs)
    for i in (0, 1, 3):
        assert rel(y[i], exact(gs[i])) <= allowed(gs[i], dt), i
    assert not y[2].any()
    assert all(torch.isnan(y[i]).all() for i in (4, 5, 6))
    zero = Orthogonalizer([(30, 40)] * 2, dt, eps=0.0)([gs[2], gs[1]])
    assert torch.isnan(zero[0]).all() and rel(zero[1], exact(gs[1], eps=0.0)) <= allowed(gs[1], dt)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(200, 300), (420, 150), (140, 5000), (131, 131), (64, 900)])
@pytest.mark.parametrize("dtype,result", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16")])
def test_special_values_tile_by_tile(shape, dtype, result):
    """The same where a matrix is made tile by tile, its square product in parts or not: small and large norms, zeros, one value that is not finite at either
    end; neighbours keep their bits."""
    dt = DTYPES[dtype]
    base = gradient(shape, torch.float32, 4, "noise") * 1e3
    top, low = (1e3, 1e-2) if dt == torch.float16 else (1e36, 1e-30)
    gs = [(base * top).to(dt), (base * low).to(dt), torch.zeros(shape, device="cuda", dtype=dt)] + [base.to(dt).clone() for _ in range(4)]
    want = Orthogonalizer([shape], dt, result_dtypes=DTYPES[result])([gs[3]])[0]
    gs[4][0, 0] = math.nan
    gs[5][-1, -1] = math.inf
    gs[6][shape[0] // 2, shape[1] - 1] = -math.inf
    y = Orthogonalizer([shape] * 7, dt, result_dtypes=DTYPES[result])(gs)
    for i in (0, 1, 3):
        assert rel(y[i], exact(gs[i])) <= allowed(gs[i], DTYPES[result]), i
    assert not y[2].any() and rel(y[3], want.double()) <= 2 * allowed(gs[3], DTYPES[result])
    assert all(torch.isnan(y[i]).all() for i in (4, 5, 6))
    zero = Orthogonalizer([shape] * 2, dt, eps=0.0, result_dtypes=DTYPES[result])([gs[2], gs[1]])
    assert torch.isnan(zero[0]).all() and rel(zero[1], exact(gs[1], eps=0.0)) <= allowed(gs[1], DTYPES[result])


@pytest.mark.gpu
def test_same_bits_wherever_it_stands():
    """A matrix has the same result again, and beside others of its shape."""
    g, other = gradient((300, 400), torch.bfloat16, 1), gradient((300, 400), torch.bfloat16, 2)
    plan = Orthogonalizer([(300, 400)] * 4, torch.bfloat16)
    a = plan([g, other, other, g])
    b = plan([other, g, g, other])
    assert torch.equal(a[0], a[3]) and torch.equal(a[0], b[1]) and torch.equal(b[1], b[2]) and torch.equal(a[1], b[0])


@pytest.mark.gpu
def test_streams_and_graphs():
    shapes = [(200, 300), (64, 576), (500, 140)]
    gs = [gradient(s, torch.bfloat16, i) for i, s in enumerate(shapes)]
    plan = Orthogonalizer(shapes, torch.bfloat16)
    want = plan(gs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = plan([g * 1 for g in gs])
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    cap = torch.cuda.Stream()
    own = Orthogonalizer(shapes, torch.bfloat16, stream=cap.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    out = [torch.empty_like(g) for g in gs]
    with torch.cuda.graph(graph, stream=cap):
        own(gs, out)
    for i, g in enumerate(gs):
        g.copy_(gradient(g.shape, torch.bfloat16, 50 + i))
    torch.cuda.synchronize()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, plan(gs)))


@pytest.mark.gpu
def test_two_plans_at_once():
    """On two streams, beside a loss on a third: all their blocks have to share the SMs."""
    shapes = [(300, 500), (140, 900), (100, 64)]
    kinds = [torch.bfloat16, torch.float32]
    streams = [torch.cuda.Stream() for _ in range(3)]
    gs = [[gradient(s, k, i + 10 * q) for i, s in enumerate(shapes)] for q, k in enumerate(kinds)]
    want = [Orthogonalizer(shapes, k)(g) for k, g in zip(kinds, gs)]
    x, w, t = torch.randn((2000, 128), device="cuda").bfloat16(), torch.randn((5000, 128), device="cuda").bfloat16(), torch.randint(5000, (2000,), device="cuda")
    loss = linear_cross_entropy_forward(x, w, t)[0]
    plans = [Orthogonalizer(shapes, k, stream=s.cuda_stream) for k, s in zip(kinds, streams)]
    torch.cuda.synchronize()
    got, losses = [[], []], []
    for _ in range(10):
        for q in range(2):
            with torch.cuda.stream(streams[q]):
                got[q].append(plans[q](gs[q]))
        with torch.cuda.stream(streams[2]):
            losses.append(linear_cross_entropy_forward(x, w, t)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(v, loss) for v in losses)
    for q in range(2):
        assert all(torch.equal(a, b) for run in got[q] for a, b in zip(run, want[q]))


@pytest.mark.gpu
def test_what_a_call_writes_counts_as_changed():
    w = gradient((20, 30), torch.float32, 1).requires_grad_()
    y = (w * w).sum()
    with torch.no_grad():
        Orthogonalizer([(20, 30)])([w], [w])
    with pytest.raises(RuntimeError):
        y.backward()


@pytest.mark.gpu
def test_results_by_iterators():
    """What is returned can be read again: the lists of what iterators gave, otherwise the very objects."""
    shapes = [(20, 30), (9, 4)]
    gs = [[gradient(s, torch.float32, 10 * k + i) for i, s in enumerate(shapes)] for k in range(2)]
    one, two = Orthogonalizer(shapes), Orthogonalizer(shapes, num_rows=2)
    want = two(gs)
    for make in (lambda o: o, tuple, iter, lambda o: (t for t in o), lambda o: dict(enumerate(o)).values()):
        out = [[torch.empty_like(g) for g in row] for row in gs]
        given = make(out[0])
        got = one(gs[0], given)
        assert got is given or not isinstance(given, (list, tuple))
        assert all(a is b for a, b in zip(list(got), out[0])) and len(list(got)) == 2
        for outer in (list, iter):
            got = two(gs, outer([make(row) for row in out]))
            assert len(got) == 2 and all(a is b and torch.equal(b, c) for r, o, w in zip(got, out, want) for a, b, c in zip(list(r), o, w)) and len(list(got[1])) == 2


@pytest.mark.gpu
def test_bad_calls_are_refused():
    plan = Orthogonalizer([(8, 6), (4, 4, 3)])
    a, b = torch.ones((8, 6), device="cuda"), torch.ones((4, 4, 3), device="cuda")
    for args in (([a],), ([a, b, b],), (a,), ([a, b.cpu()],), ([a.half(), b],), ([a.t().contiguous().t(), b],), ([torch.ones((6, 8), device="cuda"), b],),
                 ([a[:1].expand(8, 6), b],), ([a, b], [a]), ([a, b], [a, b.double()]), ([[a, b], [a, b]],), ([a, 3],)):
        with pytest.raises((ValueError, TypeError)):
            plan(*args)
    plan([a, b])
    plan.close()
    with pytest.raises(sb.SaeError):
        plan([a, b])
    plan.close()
    with pytest.raises(sb.SaeError):
        Orthogonalizer([(4, 4)], coefficients=(40.0, 0.0, 0.0))
