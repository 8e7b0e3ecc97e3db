"""The orthogonalised update against a plain implementation in 64 bits.

Tolerances (set before the first run).  fp32: operands of 22 bits and fp32 sums, an error of about 2^-22 per product; a step lengthens
errors in the directions of small singular values by up to a = 3.44 while it lengthens X by about as much: 1e-5 relative L2 of the whole.
bf16: the output's rounding (2^-9 at most) and products of 11-bit operands (2^-12 each, a handful of them carried through): 6e-3.
"""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-5, "bf16": 6e-3}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ABC = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def inst():
    import paper_2206_08482_amd as g
    h = g.gmi_create(None, 0)
    yield h
    g.gmi_destroy(h)


def steps64(u, steps, eps=1e-7):
    x = u / (u.norm() + eps)
    for _ in range(steps):
        s = x @ x.T
        x = ABC[0] * x + (ABC[1] * s + ABC[2] * (s @ s)) @ x
    return x


def layout(shapes, gap=3, lead=1):
    out, at = [], lead
    for r, c in shapes:
        out.append((r, c, at))
        at += r * c + gap
    return out, at


def gradient(shapes, total, mats, type_, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    v = torch.full((total,), 7.0, dtype=torch.float64)
    for r, c, o in mats:
        k = min(3, r, c)
        g = torch.randn(r, k, generator=gen, dtype=torch.float64) @ torch.randn(k, c, generator=gen, dtype=torch.float64)
        g = g + torch.randn(r, c, generator=gen, dtype=torch.float64)
        v[o:o + r * c] = (scale * g).flatten()
    return v.to(type_).cuda()


def part(v, m):
    r, c, o = m
    return v[o:o + r * c].reshape(r, c)


def outside(total, mats):
    keep = torch.ones(total, dtype=torch.bool)
    for r, c, o in mats:
        keep[o:o + r * c] = False
    return keep


def rel(x, y):
    return float((x.double().cpu() - y).norm() / y.norm())


SHAPES = [[(1, 1)], [(1, 9)], [(9, 1)], [(2, 2), (3, 5), (5, 3)], [(8, 8)], [(64, 64)], [(65, 130)], [(200, 33)], [(211, 512)], [(512, 211)],
          [(256, 128), (17, 300), (128, 128), (100, 1000), (1, 40)], [(600, 600)], [(32, 2000), (2000, 32)]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shapes", SHAPES, ids=str)
def test_orthogonalize(inst, shapes, dtype):
    import paper_2206_08482_amd as g
    mats, total = layout(shapes)
    src = gradient(shapes, total, mats, TYPES[dtype], 1)
    dst = torch.full_like(src, 5.0)
    h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
    for steps in (1, 5):
        torch.cuda.synchronize()
        g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams(steps=steps))
        g.gmi_sync(inst)
        for m in mats:
            want = steps64(part(src, m).double().cpu(), steps)
            assert rel(part(dst, m), want) <= TOL[dtype], (m, steps)
        assert (dst.cpu()[outside(total, mats)] == 5.0).all()
    # in place, and again: the same bits
    again = src.clone()
    torch.cuda.synchronize()
    g.muon_orthogonalize(inst, h, again, again, g.muon_hparams(steps=5))
    g.gmi_sync(inst)
    for m in mats:
        assert torch.equal(part(again, m), part(dst, m))
    g.gmi_muon_destroy(h)


@pytest.mark.parametrize("shape", [(1100, 4100), (4100, 1100), (2100, 2060)])
def test_large_tiles(inst, shape):
    import paper_2206_08482_amd as g
    mats, total = layout([shape], lead=0)
    for dtype in ("f32", "bf16"):
        src = gradient([shape], total, mats, TYPES[dtype], 2)
        dst = torch.empty_like(src)
        h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
        torch.cuda.synchronize()
        g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams(steps=3))
        g.gmi_sync(inst)
        u = part(src, mats[0]).double()
        want = (steps64(u, 3) if shape[0] <= shape[1] else steps64(u.T.contiguous(), 3).T).cpu()
        assert rel(part(dst, mats[0]), want) <= TOL[dtype]
        g.gmi_muon_destroy(h)


@pytest.mark.parametrize("shapes", [[(4096, 4096)], [(3000, 3000), (300, 100), (60, 2000)], [(17, 3568), (256, 256)], [(2119, 143)]], ids=str)
def test_tiles_of_192_and_divided_contractions(inst, shapes):
    import paper_2206_08482_amd as g
    mats, total = layout(shapes, lead=0)
    for dtype in ("f32", "bf16"):
        src = gradient(shapes, total, mats, TYPES[dtype], 7)
        dst = torch.full_like(src, 5.0)
        h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
        torch.cuda.synchronize()
        g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams(steps=2))
        g.gmi_sync(inst)
        for m in mats:
            u = part(src, m).double()
            want = (steps64(u, 2) if m[0] <= m[1] else steps64(u.T.contiguous(), 2).T).cpu()
            assert rel(part(dst, m), want) <= TOL[dtype], m
        assert (dst.cpu()[outside(total, mats)] == 5.0).all()
        g.gmi_muon_destroy(h)


def test_a_step_in_a_graph(inst):
    """A captured step, replayed on restored state with other work in between, gives what the call gives."""
    import paper_2206_08482_amd as g
    shapes = [(128, 256), (300, 90)]
    mats, total = layout(shapes)
    gen = torch.Generator().manual_seed(3)
    params0, moments0 = (torch.randn(total, generator=gen).cuda() for _ in range(2))
    grad = gradient(shapes, total, mats, torch.float32, 8)
    params, moments = params0.clone(), moments0.clone()
    h, hp = g.gmi_muon_bind(inst, mats, g.DTYPE_F32), g.muon_hparams()
    stream = torch.cuda.ExternalStream(g.gmi_stream(inst))
    torch.cuda.synchronize()
    g.muon_update(inst, h, params, moments, grad, hp)
    g.gmi_sync(inst)
    want = params.clone(), moments.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        g.muon_update(inst, h, params, moments, grad, hp)
    for _ in range(3):
        params.copy_(params0)
        moments.copy_(moments0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(params, want[0]) and torch.equal(moments, want[1])
    g.gmi_muon_destroy(h)


def test_singular_values_become_one(inst):
    """With the usual coefficients five steps bring every singular value that starts above 0.01 of the norm into 0.6 .. 1.25."""
    import paper_2206_08482_amd as g
    gen = torch.Generator().manual_seed(5)
    q, _ = torch.linalg.qr(torch.randn(96, 96, generator=gen, dtype=torch.float64))
    p, _ = torch.linalg.qr(torch.randn(160, 96, generator=gen, dtype=torch.float64))
    src = (q @ torch.diag(torch.linspace(0.2, 1.0, 96, dtype=torch.float64)) @ p.T).float().cuda()
    dst = torch.empty_like(src)
    h = g.gmi_muon_bind(inst, [(96, 160, 0)], g.DTYPE_F32)
    torch.cuda.synchronize()
    g.muon_orthogonalize(inst, h, src.view(-1), dst.view(-1), g.muon_hparams())
    g.gmi_sync(inst)
    s = torch.linalg.svdvals(dst.double().cpu())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25
    g.gmi_muon_destroy(h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-20, 1e-6, 1e15])
def test_scales_of_the_gradient(inst, scale, dtype):
    """The result depends on the gradient's size only through eps; squares of large values must not overflow."""
    import paper_2206_08482_amd as g
    mats, total = layout([(40, 90), (90, 40)])
    src = gradient(None, total, mats, TYPES[dtype], 3, scale)
    dst = torch.empty_like(src)
    h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
    torch.cuda.synchronize()
    g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams())
    g.gmi_sync(inst)
    for m in mats:
        want = steps64(part(src, m).double().cpu(), 5)
        got = part(dst, m).double().cpu()
        # of 1e-20 hardly anything is left after the division by eps: there the fp16 planes' smallest steps bound the error
        assert float((got - want).norm()) <= TOL[dtype] * float(want.norm()) + 1e-9 * math.sqrt(40 * 90), (m, scale)
    g.gmi_muon_destroy(h)


def test_zero_and_not_finite(inst):
    import paper_2206_08482_amd as g
    mats, total = layout([(40, 50), (50, 40), (70, 70), (64, 100)])
    for dtype in ("f32", "bf16"):
        src = gradient(None, total, mats, TYPES[dtype], 4)
        part(src, mats[0]).zero_()
        part(src, mats[1])[3, 4] = float("inf")
        part(src, mats[2])[69, 69] = float("nan")
        dst = torch.empty_like(src)
        h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
        torch.cuda.synchronize()
        g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams())
        g.gmi_sync(inst)
        assert (part(dst, mats[0]) == 0).all()
        assert torch.isnan(part(dst, mats[1])).all() and torch.isnan(part(dst, mats[2])).all()
        assert rel(part(dst, mats[3]), steps64(part(src, mats[3]).double().cpu(), 5)) <= TOL[dtype]
        g.gmi_muon_destroy(h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("lead", [0, 1])
def test_update(inst, lead, nesterov, dtype):
    import paper_2206_08482_amd as g
    shapes = [(64, 128), (200, 48), (33, 65), (256, 256)]
    mats, total = layout(shapes, gap=8 if lead == 0 else 3, lead=lead)
    gen = torch.Generator().manual_seed(9)
    params, moments = (torch.randn(total, generator=gen).cuda() for _ in range(2))
    grad = gradient(shapes, total, mats, TYPES[dtype], 6)
    hp = dict(lr=0.05, momentum=0.9, weight_decay=0.1, nesterov=nesterov)
    h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
    p1, m1 = torch.full_like(params, 3.0), torch.full_like(params, 4.0)
    torch.cuda.synchronize()
    g.muon_update(inst, h, params, moments, grad, g.muon_hparams(**hp), p1, m1)
    p2, m2 = params.clone(), moments.clone()
    torch.cuda.synchronize()
    g.muon_update(inst, h, p2, m2, grad, g.muon_hparams(**hp))
    g.gmi_sync(inst)
    keep = outside(total, mats)
    assert (p1.cpu()[keep] == 3.0).all() and (m1.cpu()[keep] == 4.0).all()
    assert torch.equal(p2.cpu()[keep], params.cpu()[keep]) and torch.equal(m2.cpu()[keep], moments.cpu()[keep])
    for m in mats:
        gg, mm, pp = (part(v, m).double().cpu() for v in (grad, moments, params))
        new = 0.9 * mm + gg
        u = gg + 0.9 * new if nesterov else new
        step = 0.05 * math.sqrt(max(1.0, m[0] / m[1])) * steps64(u, 5)
        want = (1 - 0.05 * 0.1) * pp - step
        assert torch.equal(part(p1, m), part(p2, m)) and torch.equal(part(m1, m), part(m2, m))
        assert rel(part(m1, m), new) <= 1e-6
        # the step's own error, and the rounding of parameters of size 1 to fp32
        assert float((part(p1, m).double().cpu() - want).norm()) <= TOL[dtype] * float(step.norm()) + 2e-7 * float(pp.norm())
    g.gmi_muon_destroy(h)


def test_refusals(inst):
    import paper_2206_08482_amd as g

    def refused(code, f, *a):
        with pytest.raises(g.GmiError) as e:
            f(*a)
        assert e.value.code == code, e.value

    f32 = g.DTYPE_F32
    refused(g.ERR_BAD_SHAPE, g.gmi_muon_bind, inst, [], f32)
    refused(g.ERR_BAD_SHAPE, g.gmi_muon_bind, inst, [(0, 4, 0)], f32)
    refused(g.ERR_BAD_SHAPE, g.gmi_muon_bind, inst, [(4, 40000, 0)], f32)
    refused(g.ERR_BAD_SHAPE, g.gmi_muon_bind, inst, [(4, 4, -1)], f32)
    refused(g.ERR_INVALID_ARG, g.gmi_muon_bind, inst, [(4, 4, 0), (4, 4, 15)], f32)
    refused(g.ERR_UNSUPPORTED, g.gmi_muon_bind, inst, [(4, 4, 0)], 9)
    refused(g.ERR_BAD_HANDLE, g.gmi_muon_bind, 0, [(4, 4, 0)], f32)
    h = g.gmi_muon_bind(inst, [(4, 4, 0)], f32)
    a, b, c, d = (torch.zeros(64, device="cuda") for _ in range(4))
    torch.cuda.synchronize()
    hp = g.muon_hparams
    refused(g.ERR_INVALID_ARG, g.muon_orthogonalize, inst, h, a, b, hp(steps=0))
    refused(g.ERR_INVALID_ARG, g.muon_orthogonalize, inst, h, a, b, hp(steps=65))
    refused(g.ERR_INVALID_ARG, g.muon_orthogonalize, inst, h, a, b, hp(eps=0.0))
    refused(g.ERR_INVALID_ARG, g.muon_orthogonalize, inst, h, a, a[4:], hp())
    refused(g.ERR_INVALID_ARG, g.muon_update, inst, h, a, b, c, hp(), b, d)
    refused(g.ERR_INVALID_ARG, g.muon_update, inst, h, a, b, c, hp(), c, d)
    refused(g.ERR_INVALID_ARG, g.muon_update, inst, h, a, a, c, hp())
    lib = g._lib
    import ctypes
    refused(g.ERR_INVALID_ARG, lambda: g._check(lib.muon_orthogonalize(inst, h, None, b.data_ptr(), ctypes.byref(hp()))))
    refused(g.ERR_INVALID_ARG, lambda: g._check(lib.muon_orthogonalize(inst, h, a.data_ptr() + 2, b.data_ptr(), ctypes.byref(hp()))))
    refused(g.ERR_INVALID_ARG, lambda: g._check(lib.muon_orthogonalize(inst, h, a.data_ptr(), b.data_ptr(), None)))
    refused(g.ERR_BAD_HANDLE, lambda: g._check(lib.muon_orthogonalize(inst, inst, a.data_ptr(), b.data_ptr(), ctypes.byref(hp()))))
    with pytest.raises(ValueError):
        g.muon_orthogonalize(inst, h, a[:8], b, hp())
    with pytest.raises(ValueError):
        g.muon_orthogonalize(inst, h, a.half(), b.half(), hp())
    g.gmi_muon_destroy(h)


def steps64_of(u, steps, abc, eps=1e-7):
    x = u / (u.norm() + eps)
    for _ in range(steps):
        s = x @ x.T
        x = abc[0] * x + (abc[1] * s + abc[2] * (s @ s)) @ x
    return x


# entries of the first size or so; the norm is some 60 times that
# (coefficients for 14 steps: ones that bring the singular values to 1 and hold them there)
@pytest.mark.parametrize("steps,abc", [(1, ABC), (5, ABC), (14, (2.0, -1.5, 0.5))], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,eps", [(1e-6, 1e-7), (1e-9, 1e-7), (1e-12, 1e-7), (1e-14, 1e-7), (1e-18, 1e-7), (1e-24, 1e-7), (1e-3, 1.0), (3.0, 1e4),
                                      (1e-20, 1e-20), (6e36, 1e-7), (3e37, 1e-7)])
def test_gradients_of_any_size_relative_to_the_result(inst, size, eps, dtype, steps, abc):
    """However little the division by |G| + eps leaves, and where the norm is beyond the type: the same relative error."""
    import paper_2206_08482_amd as g
    mats, total = layout([(40, 90), (90, 40)])
    src = gradient(None, total, mats, TYPES[dtype], 3, size / 3)
    assert torch.isfinite(src).all()
    dst = torch.empty_like(src)
    h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
    torch.cuda.synchronize()
    g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams(steps=steps, eps=eps, a=abc[0], b=abc[1], c=abc[2]))
    g.gmi_sync(inst)
    for m in mats:
        want = steps64_of(part(src, m).double().cpu(), steps, abc, float(torch.tensor(eps)))
        assert rel(part(dst, m), want) <= TOL[dtype], m
    g.gmi_muon_destroy(h)


def concentrated(r, c, type_, seed):
    """A matrix of rank one: its one singular value is its norm."""
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(r, 1, generator=gen, dtype=torch.float64) @ torch.randn(1, c, generator=gen, dtype=torch.float64)).to(type_)


# (coefficients, steps): singular values that reach 20, 400; 47 and, from there, 5e6; 60 after 100 at small ones
COEFFICIENTS = [((20.0, 0.0, 0.0), 2), ((20.0, 0.0, 0.0), 3), ((3.4445, -50.0, 0.0), 1), ((3.4445, -50.0, 0.0), 2), ((100.0, -50.0, 10.0), 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("abc,steps", COEFFICIENTS, ids=str)
def test_coefficients_that_lengthen(inst, abc, steps, dtype):
    """The largest singular value there can be, the norm itself.  With a = 3.4445, b = -50 a step multiplies relative errors by up to 3; the
    tolerances hold roundings of the planes by 4 (2^-12 each, 2^-22 in fp32) several times over, twice so for two such steps."""
    import paper_2206_08482_amd as g
    shapes = [(1, 1), (33, 70), (130, 20), (200, 200)]
    mats, total = layout(shapes)
    src = torch.zeros(total, dtype=TYPES[dtype])
    for i, (r, c, o) in enumerate(mats):
        src[o:o + r * c] = concentrated(r, c, TYPES[dtype], 20 + i).flatten()
    src = src.cuda()
    dst = torch.full_like(src, 5.0)
    h = g.gmi_muon_bind(inst, mats, g.dtype_code(dtype))
    torch.cuda.synchronize()
    g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams(steps=steps, a=abc[0], b=abc[1], c=abc[2]))
    g.gmi_sync(inst)
    for m in mats:
        want = steps64_of(part(src, m).double().cpu(), steps, abc)
        assert rel(part(dst, m), want) <= TOL[dtype] * (2 if steps == 2 else 1), m
    g.gmi_muon_destroy(h)


def test_coefficients_beyond_the_planes_are_refused(inst):
    import paper_2206_08482_amd as g
    h = g.gmi_muon_bind(inst, [(4, 4, 0)], g.DTYPE_F32)
    src = torch.eye(4, device="cuda").flatten()
    dst, moments, params = torch.full_like(src, 5.0), torch.zeros_like(src), torch.ones_like(src)
    torch.cuda.synchronize()
    nan = float("nan")
    for kw in (dict(a=2000.0, b=0.0, c=0.0, steps=3), dict(b=-50.0, c=0.0, steps=4), dict(a=1e30), dict(c=1e38), dict(a=nan), dict(b=nan), dict(c=float("inf"))):
        hp = g.muon_hparams(**kw)
        for call in (lambda: g.muon_orthogonalize(inst, h, src, dst, hp), lambda: g.muon_update(inst, h, params, moments, src, hp)):
            with pytest.raises(g.GmiError) as e:
                call()
            assert e.value.code == g.ERR_INVALID_ARG, kw
    g.gmi_sync(inst)
    assert (dst == 5.0).all() and (params == 1.0).all() and (moments == 0.0).all()
    g.muon_orthogonalize(inst, h, src, dst, g.muon_hparams(a=2000.0, b=0.0, c=0.0, steps=1))      # the last step's result is not kept in planes
    g.gmi_sync(inst)
    assert torch.allclose(dst, 1000.0 * src, rtol=1e-5)
    g.gmi_muon_destroy(h)


@pytest.mark.parametrize("cus", [8, 104])
def test_instances_of_some_compute_units(inst, cus):
    """Tiles and divisions of the contraction are planned for the binding's instance; another one may call it."""
    import paper_2206_08482_amd as g
    from paper_2206_08482_amd.instances import cu_masks
    few = g.gmi_create(cu_masks(256, [cus])[0])
    shapes = [(600, 600), (17, 3568), (211, 512), (90, 40)]
    mats, total = layout(shapes)
    for dtype in ("f32", "bf16"):
        src = gradient(shapes, total, mats, TYPES[dtype], 12)
        h = g.gmi_muon_bind(few, mats, g.dtype_code(dtype))
        for caller in (few, inst):
            dst = torch.full_like(src, 5.0)
            torch.cuda.synchronize()
            g.muon_orthogonalize(caller, h, src, dst, g.muon_hparams(steps=3))
            g.gmi_sync(caller)
            for m in mats:
                assert rel(part(dst, m), steps64(part(src, m).double().cpu(), 3)) <= TOL[dtype], m
            assert (dst.cpu()[outside(total, mats)] == 5.0).all()
        g.gmi_muon_destroy(h)
    g.gmi_destroy(few)
