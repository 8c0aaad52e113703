"""The operators around attention on the GPU against plain implementations in 64 bits.

Tolerances are elementwise bounds, formed from the reference's own magnitudes before
anything runs. A value rounded to its type is off by at most u |value| (u, the unit
roundoff, is 2^-24, 2^-8 and 2^-11 for fp32, bf16 and fp16; below fp16's normal range by
2^-25), and an fp32 sum by at most k 2^-24 times the sum of magnitudes of what it adds, k
the roundings on the way of one number through it.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.fixture(scope="module")
def bev(torch):
    import paper_2205_13542_amd as bev
    bev._map_binding.load()
    return bev


def _dtype(torch, name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _u(name):
    return {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[name]


def _tiny(name):
    """Half the spacing of the type's subnormal numbers."""
    return {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}[name]


def _check(what, got, ref, tol):
    got = got.double()
    assert got.shape == ref.shape, what
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float(((got - ref).abs() / tol.clamp(min=1e-300)).max()):.3g} of the bound")


def _normal(torch, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *shape, s=1.0: s * torch.randn(shape, generator=gen, device="cuda")


def _over(torch, number, t):
    """number / t in one rounding (with a plain number torch multiplies by a reciprocal)."""
    return torch.full_like(t, number) / t


# ---------------------------------------------------------------- RMS norm

# Roundings of a number on its way through a row's sum: at most 32 products of a lane, one
# after the other, six halvings over a wave and two over its workgroup.
ROW = 40
# The same through a weight's gradient: at least 8 rows of a lane (more only of over 2048 * 32
# rows), six halvings, four waves, 32 parts of a lane and six halvings.
COLUMN = 56


def _rms_reference(torch, x, residual, w, eps, dy, dsum, x_type, y_type, w_type):
    x, w = x.double(), w.double()
    h = x if residual is None else x + residual.double()
    rstd = 1 / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    u, y = h * rstd, h * rstd * w
    # h is rounded once (a sum of fp32), its square's sum ROW times, rstd by half of that and by 3 of its
    # own, the two products that follow once each
    rel = (2 + ROW / 2 + 3 + 2) * U32
    out = {"y": (y, rel * y.abs() + _u(y_type) * y.abs() + _tiny(y_type)),
           "total": (h, (U32 + _u(x_type)) * h.abs() + _tiny(x_type))}
    if dy is None:
        return out
    dy = dy.double()
    du = rel * u.abs()
    e = dy * w
    m = (e * u).mean(-1, keepdim=True)
    dm = (e.abs() * du + (ROW + 3) * U32 * (e * u).abs()).mean(-1, keepdim=True) + 2 * U32 * m.abs()
    dh = rstd * (e - u * m)
    tol = rstd * (2 * U32 * e.abs() + du * m.abs() + u.abs() * dm + 2 * U32 * (u * m).abs()) + rel * dh.abs()
    if dsum is not None:
        dh = dh + dsum.double()
        tol = tol + U32 * dh.abs()
    out["dx"] = (dh, tol + 1.01 * _u(x_type) * dh.abs() + _tiny(x_type))
    flat = (dy * u).flatten(0, -2)
    size = (dy.abs() * du + COLUMN * U32 * (dy * u).abs()).flatten(0, -2).sum(0)
    dw = flat.sum(0)
    out["dw"] = (dw, size + 1.01 * _u(w_type) * dw.abs() + _tiny(w_type))
    return out


RMS_CASES = [
    # shape, channels left of a slice, residual, x, y, weight
    ((1, 1), 0, False, "f32", "f32", "f32"),
    ((1, 256), 0, True, "bf16", "bf16", "f32"),
    ((3, 5, 80), 0, True, "bf16", "bf16", "bf16"),
    ((7, 64), 16, False, "f16", "f16", "f16"),
    ((600, 256), 0, True, "f16", "f16", "f32"),
    ((1111, 331), 0, True, "f32", "bf16", "f32"),           # one element to an access
    ((517, 66), 3, True, "bf16", "f32", "f32"),
    ((300, 130), 0, False, "f16", "bf16", "f16"),           # two
    ((20000, 80), 0, True, "bf16", "bf16", "f32"),          # many rows to a workgroup
    ((70001, 24), 8, False, "f32", "f32", "f32"),
    ((8200, 1024), 0, False, "bf16", "bf16", "f32"),        # two accesses of a wave
    ((8193, 516), 0, True, "f32", "f32", "f32"),            # four
    ((8192, 300), 1, True, "bf16", "bf16", "f32"),          # eight, one or two at a time
    ((100, 2048), 0, True, "bf16", "f16", "f32"),           # a workgroup to a row
    ((33, 4100), 0, True, "f32", "f32", "f32"),
    ((33, 1027), 0, False, "bf16", "bf16", "f32"),
    ((5, 8192), 0, True, "f32", "f32", "f32"),              # the most channels
    ((5, 8190), 0, True, "f16", "f16", "f32"),
    ((3, 8191), 2, False, "bf16", "bf16", "f32"),
    # rows shorter than an access, and of one and a bit
    ((50, 5), 0, True, "bf16", "f32", "f32"),
    ((2000, 3), 1, True, "f32", "bf16", "bf16"),
    ((1500, 9), 0, True, "f16", "f32", "f32"),
    ((70, 5), 0, False, "f32", "f16", "f32"),
    ((1025, 100), 0, True, "bf16", "bf16", "f32"),
    ((1024, 2047), 3, True, "f16", "f32", "bf16"),
]


@pytest.mark.parametrize("shape,left,residual,x_type,y_type,w_type", RMS_CASES)
def test_rms_norm(torch, bev, shape, left, residual, x_type, y_type, w_type):
    normal = _normal(torch, 1)
    C = shape[-1]
    dtype = _dtype(torch, x_type)
    loud = torch.exp(normal(*shape[:-1], 1))
    x = normal(*shape[:-1], left + C).to(dtype)[..., left:].requires_grad_()
    r = (normal(*shape) * loud).to(dtype).requires_grad_() if residual else None
    w = (1 + normal(C, s=0.2)).to(_dtype(torch, w_type)).requires_grad_()
    dy = normal(*shape).to(_dtype(torch, y_type))
    dsum = normal(*shape).to(dtype) if residual else None
    out = _dtype(torch, y_type)
    if residual:
        y, total = bev.rms_norm_add(x, r, w, eps=1e-5, out_dtype=out)
        dx, dr, dw = torch.autograd.grad((y, total), (x, r, w), (dy, dsum))
        assert torch.equal(dx, dr)
    else:
        y, total = bev.rms_norm(x, w, eps=1e-5, out_dtype=out), None
        dx, dw = torch.autograd.grad(y, (x, w), dy)
    ref = _rms_reference(torch, x.detach(), None if r is None else r.detach(), w.detach(), 1e-5, dy, dsum, x_type,
                         y_type, w_type)
    got = {"y": y.detach(), "dx": dx, "dw": dw}
    if residual:
        got["total"] = total.detach()
    for name, value in got.items():
        assert value.is_contiguous()
        _check(name, value, *ref[name])
    with torch.no_grad():
        again = bev.rms_norm_add(x, r, w, eps=1e-5, out_dtype=out)[0] if residual else bev.rms_norm(
            x, w, eps=1e-5, out_dtype=out)
    assert torch.equal(again, y)


def test_rms_norm_without_weight_or_one_result(torch, bev):
    normal = _normal(torch, 2)
    x, r, dy, dsum = (normal(9, 40) for _ in range(4))
    ones = torch.ones(40, device="cuda")
    assert torch.equal(bev.rms_norm(x), bev.rms_norm(x, ones))
    x.requires_grad_(), r.requires_grad_()
    w = ones.clone().requires_grad_()
    y, total = bev.rms_norm_add(x, r, w)
    both = torch.autograd.grad((y, total), (x, r, w), (dy, torch.zeros_like(dsum)), retain_graph=True)
    alone = torch.autograd.grad(y, (x, r, w), dy, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(both, alone))
    dx, dr, dw = torch.autograd.grad(total, (x, r, w), dsum)
    assert torch.equal(dx, dsum) and torch.equal(dr, dsum) and not dw.any()
    y, total = bev.rms_norm_add(x.detach(), r)      # one leaf alone
    got, = torch.autograd.grad((y, total), (r,), (dy, dsum))
    y2, total2 = bev.rms_norm_add(x, r.detach(), w.detach())
    ref, = torch.autograd.grad((y2, total2), (x,), (dy, dsum))
    assert torch.equal(got, ref)


@pytest.mark.parametrize("channels", [24, 1030, 8192])
def test_rms_norm_of_any_size(torch, bev, channels):
    """Squares past fp32's range, rows of zeros, infinities and NaN in rows of their own."""
    normal = _normal(torch, 3)
    x = normal(8, channels)
    x[1] *= 2.0 ** 100
    x[2] *= 2.0 ** -100
    x[3] = 0
    x[4, 3] = math.inf
    x[5, 7] = math.nan
    x[6] *= 2.0 ** 64
    y = bev.rms_norm(x, eps=0.0)
    ref = x.double() / x.double().square().mean(1, keepdim=True).sqrt()
    fine = [0, 1, 2, 6, 7]
    _check("y", y[fine], ref[fine], 32 * U32 * ref[fine].abs())
    assert y[5].isnan().all() and y[4, 3].isnan() and (y[4, :3] == 0).all()
    assert y[3].isnan().all()                               # 0 / 0 with eps of 0
    assert not bev.rms_norm(x)[3].any()                     # and 0 with any other
    small = bev.rms_norm(x[2:3], eps=1e-6)
    _check("small", small, x[2:3].double() * 1000, 1e-6 * x[2:3].double().abs() * 1000)
    held, scale = bev.rms_norm_int8(x, eps=1e-6)
    assert scale[4:6].isnan().all() and not held[3:6].any() and scale[3] == 0
    x[2] *= 2.0 ** -30                                      # below fp32's normal numbers
    held, scale = bev.quantize_int8(x)
    z = x[2] * 2.0 ** 64
    assert torch.equal(held[2], torch.round(z * _over(torch, 127, z.abs().max())).to(torch.int8))


@pytest.mark.parametrize("shape,left,residual,x_type,y_type,w_type", RMS_CASES)
def test_rms_norm_int8(torch, bev, shape, left, residual, x_type, y_type, w_type):
    normal = _normal(torch, 4)
    C = shape[-1]
    dtype = _dtype(torch, x_type)
    x = normal(*shape[:-1], left + C).to(dtype)[..., left:]
    r = normal(*shape).to(dtype) if residual else None
    w = (1 + normal(C, s=0.2)).to(_dtype(torch, w_type))
    if residual:
        held, scale, total = bev.rms_norm_add_int8(x, r, w)
        assert torch.equal(total, bev.rms_norm_add(x, r, w)[1])
    else:
        held, scale = bev.rms_norm_int8(x, w)
    assert held.dtype == torch.int8 and held.shape == x.shape and scale.shape == x.shape[:-1]
    h = x.float() if r is None else x.float() + r.float()
    # every step is one correctly rounded fp32 operation, the same here and there
    z = h * w.float()
    assert torch.equal(held, torch.round(z * _over(torch, 127, z.abs().amax(-1, keepdim=True))).to(torch.int8))
    assert (held.abs().amax(-1) == 127).all()
    y, _ = _rms_reference(torch, x, r, w, 1e-6, None, None, "f32", "f32", "f32")["y"]
    _check("scale", scale, y.abs().amax(-1) / 127, (ROW / 2 + 12) * U32 * y.abs().amax(-1) / 127)
    step = scale.double()[..., None]
    _check("values", held.double() * step, y, 0.5 * step + (ROW / 2 + 16) * U32 * 127 * step)


@pytest.mark.parametrize("shape,x_type", [((1, 1), "f32"), ((5, 80), "bf16"), ((4, 33, 130), "f16"), ((300, 331), "f32"),
                                          ((2, 8193), "bf16"), ((3, 40000), "f32"), ((2, 131071), "f16")])
def test_quantize_int8(torch, bev, shape, x_type):
    x = _normal(torch, 5)(*shape).to(_dtype(torch, x_type))
    held, scale = bev.quantize_int8(x)
    top = x.float().abs().amax(-1, keepdim=True)
    assert torch.equal(held, torch.round(x.float() * _over(torch, 127, top)).to(torch.int8))
    assert torch.equal(scale, (top / torch.full_like(top, 127)).squeeze(-1))


# ---------------------------------------------------------------- product of 8-bit integers

def _held(torch, seed, rows, columns, most=127):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-most - 1, most + 1, (rows, columns), generator=gen, device="cuda", dtype=torch.int32)
    return q.to(torch.int8), torch.rand(rows, generator=gen, device="cuda") + 0.5


LINEAR_CASES = [
    # rows, channels, features, channels left of a slice of x, of w, bias, y
    (1, 1, 1, 0, 0, True, "f32"),
    (1, 1024, 4096, 0, 0, False, "bf16"),
    (1, 80, 17, 0, 0, True, "f16"),
    (7, 48, 33, 16, 0, False, "f32"),
    (16, 4096, 130, 0, 0, True, "bf16"),
    (17, 1000, 100, 0, 0, True, "f32"),
    (64, 2048, 256, 0, 16, False, "f16"),
    (65, 333, 90, 0, 0, True, "f32"),
    (300, 256, 256, 0, 0, True, "bf16"),
    (1111, 331, 517, 0, 0, True, "f32"),
    (1111, 331, 520, 5, 3, True, "bf16"),
    (700, 160, 1000, 0, 0, False, "f16"),
    (1500, 15, 900, 0, 0, True, "f32"),
    (4096, 80, 256, 0, 0, True, "bf16"),
    (20000, 80, 264, 0, 0, False, "bf16"),
    (20000, 83, 263, 0, 0, True, "f16"),
    (9000, 640, 2056, 0, 0, True, "bf16"),
    (9000, 640, 2049, 0, 0, False, "f32"),
    (8500, 700, 4100, 1, 0, True, "bf16"),
    # the largest tiles, all of them whole and the last ones in eighths
    (16384, 640, 1024, 0, 0, True, "bf16"),
    (16300, 515, 1020, 0, 2, False, "f16"),
    (16500, 528, 1000, 0, 0, True, "bf16"),
    (16390, 513, 1021, 3, 0, True, "f32"),
    # few tokens: one block of them and two, k shorter and longer than the waves' runs
    (32, 1040, 4096, 0, 0, True, "bf16"),
    (100, 3000, 300, 0, 0, False, "f32"),
    (40, 5000, 2000, 0, 0, True, "bf16"),
    (33, 129, 70, 0, 0, True, "f32"),
    (200, 1025, 1000, 0, 0, False, "bf16"),
    (250, 1056, 2000, 0, 0, True, "f16"),
    (16, 7, 40, 0, 0, True, "f32"),
    (700, 2000, 777, 0, 0, True, "f32"),        # tiles of 64, a k that divides nothing
    (2500, 300, 1100, 0, 0, False, "bf16"),
    (33000, 443, 509, 0, 0, True, "bf16"),      # 128 x 128 and 128 x 64 of rows that go through the registers
    (33000, 203, 509, 0, 0, True, "f16"),
    (16400, 512, 1001, 0, 0, True, "f16"),      # rows of y at any alignment, the last of it in part
    (16400, 512, 1023, 0, 0, False, "f32"),
    (9000, 300, 1026, 0, 0, False, "f32"),
    (4100, 80, 1027, 0, 0, True, "bf16"),
    (700, 80, 1005, 0, 0, True, "bf16"),
    (16400, 715, 1001, 0, 1, True, "f16"),
    (40000, 64, 7, 0, 0, True, "bf16"),         # rows of y shorter than an access
    (140000, 64, 3, 0, 0, True, "f32"),
    (70000, 33, 1, 0, 0, False, "f16"),
    (2100, 9, 2000, 0, 0, True, "f32"),         # rows shorter than an access, in tiles of 128 x 64
]


@pytest.mark.parametrize("rows,channels,features,left,w_left,bias,y_type", LINEAR_CASES)
def test_linear_int8(torch, bev, rows, channels, features, left, w_left, bias, y_type):
    x, xs = _held(torch, 1, rows, left + channels)
    w, ws = _held(torch, 2, features, w_left + channels)
    x, w = x[:, left:], w[:, w_left:]
    b = _normal(torch, 3)(features, s=100.0) if bias else None
    ws = ws * (0.01 / channels ** 0.5)
    y = bev.linear_int8(x, xs, w, ws, b, out_dtype=_dtype(torch, y_type))
    # integers of up to 2^14 and sums of up to 2^31: exact in 64 bits
    product = (x.double() @ w.double().t().contiguous()) * xs.double()[:, None] * ws.double()
    ref = product + b.double() if bias else product
    _check("y", y, ref, 3 * U32 * product.abs() + (U32 + _u(y_type)) * ref.abs() + _tiny(y_type))
    assert torch.equal(y, bev.linear_int8(x, xs, w, ws, b, out_dtype=_dtype(torch, y_type)))


@pytest.mark.parametrize("rows,features", [(16400, 1001), (16384, 1024), (3000, 2000), (700, 1000), (60, 400)])
@pytest.mark.parametrize("channels", [530, 545, 560, 592, 597, 607, 624, 637, 715, 720, 331, 333])
def test_linear_int8_ends_of_k(torch, bev, rows, features, channels):
    """k that ends in every quarter of a stage, in rows of any alignment, for every form; and
    the same again and again."""
    x, xs = _held(torch, 6, rows, channels)
    w, ws = _held(torch, 7, features, channels)
    y = bev.linear_int8(x, xs, w, ws, out_dtype=torch.float32)
    ref = (x.double() @ w.double().t().contiguous()) * xs.double()[:, None] * ws.double()
    _check("y", y, ref, 3 * U32 * ref.abs())
    for _ in range(5):
        assert torch.equal(y, bev.linear_int8(x, xs, w, ws, out_dtype=torch.float32))


def test_linear_int8_of_the_largest_sums(torch, bev):
    """The most channels, all of the largest magnitude: sums next to 2^31."""
    K = 131071
    x = torch.full((3, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((5, K), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one = torch.ones(5, device="cuda")
    y = bev.linear_int8(x, one[:3], w, one, out_dtype=torch.float32)
    ref = x.double() @ w.double().t().contiguous()
    _check("y", y, ref, U32 * ref.abs())


def test_linear_int8_shapes_and_scales(torch, bev):
    x, xs = _held(torch, 4, 6, 32)
    w, ws = _held(torch, 5, 10, 32)
    y = bev.linear_int8(x, xs, w, ws)
    assert y.dtype == torch.bfloat16
    assert torch.equal(bev.linear_int8(x.view(2, 3, 32), xs.view(2, 3), w, ws), y.view(2, 3, 10))
    assert torch.equal(bev.linear_int8(x[0], xs[0], w, ws), y[0])
    xs[2], ws[4] = math.nan, 0.0
    y = bev.linear_int8(x, xs, w, ws, out_dtype=torch.float32)
    assert y[2].isnan().all() and not y[[0, 1, 3, 4, 5]].isnan().any() and not y[[0, 1, 3, 4, 5], 4].any()
    assert bev.linear_int8(x[:0], xs[:0], w, ws).shape == (0, 10)
    assert bev.linear_int8(x, xs, w[:0], ws[:0]).shape == (6, 0)


def test_linear_int8_leaves_the_rest_alone(torch, bev):
    """Through the C ABI, into the middle of a buffer: nothing before, between or behind is written."""
    mb = bev._map_binding
    for rows, channels, features in ((3, 64, 20), (200, 100, 150), (1000, 128, 520), (5000, 128, 1032)):
        x, xs = _held(torch, 6, rows, channels)
        w, ws = _held(torch, 7, features, channels)
        buffer = torch.full((rows * features + 64,), 7.0, device="cuda")
        mb.bevmap_linear_int8(mb.bevmap_linear(rows, channels, features, channels, channels, 0), x.data_ptr(),
                              xs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, buffer.data_ptr() + 4 * 17)
        torch.cuda.synchronize()
        y = bev.linear_int8(x, xs, w, ws, out_dtype=torch.float32)
        assert torch.equal(buffer[17:17 + rows * features].view(rows, features), y)
        assert (buffer[:17] == 7).all() and (buffer[17 + rows * features:] == 7).all()


def test_linear_int8_of_uneven_rows_leaves_the_rest_alone(torch, bev):
    """The same of 16-bit rows of any length at odd addresses, in every size of tile."""
    mb = bev._map_binding
    for rows, channels, features in ((16400, 512, 1001), (33000, 100, 259), (1111, 64, 517), (8300, 64, 1035), (40000, 64, 7)):
        x, xs = _held(torch, 6, rows, channels)
        w, ws = _held(torch, 7, features, channels)
        ws = ws * 2.0 ** -10
        buffer = torch.full((rows * features + 64,), 7.0, device="cuda", dtype=torch.bfloat16)
        mb.bevmap_linear_int8(mb.bevmap_linear(rows, channels, features, channels, channels, 1), x.data_ptr(),
                              xs.data_ptr(), w.data_ptr(), ws.data_ptr(), 0, buffer.data_ptr() + 2 * 17)
        torch.cuda.synchronize()
        y = bev.linear_int8(x, xs, w, ws)
        assert torch.equal(buffer[17:17 + rows * features].view(rows, features), y)
        assert (buffer[:17] == 7).all() and (buffer[17 + rows * features:] == 7).all()


def test_uneven_results_leave_the_rest_alone(torch, bev):
    """Through the C ABI, rows of sizes that divide nothing into the middle of buffers, at odd addresses."""
    mb = bev._map_binding
    normal = _normal(torch, 8)
    for rows, C in ((7, 5), (33, 331), (9, 1027), (5, 77)):
        x, r, w = normal(rows, C).bfloat16(), normal(rows, C).bfloat16(), normal(C)
        out = [torch.full((rows * n + 64,), 7, device="cuda", dtype=t)
               for n, t in ((C, torch.bfloat16), (C, torch.bfloat16), (C, torch.int8), (C, torch.bfloat16), (C, torch.float32))]
        total, y, held, dx, wide = out
        scale = torch.empty(rows, device="cuda")
        at = [t.data_ptr() + 17 * t.element_size() for t in out]
        n = mb.bevmap_rms(rows, C, 1, 1, 0, C, C, 1e-6)
        rstd = torch.empty(rows, device="cuda")
        mb.bevmap_rms_norm(n, x.data_ptr(), r.data_ptr(), w.data_ptr(), at[0], at[1], rstd.data_ptr())
        mb.bevmap_rms_norm_int8(n, x.data_ptr(), 0, w.data_ptr(), 0, at[2], scale.data_ptr())
        mb.bevmap_rms_norm_backward(n, r.data_ptr(), 0, x.data_ptr(), 0, w.data_ptr(), rstd.data_ptr(), at[3], 0, 0, 0)
        n = mb.bevmap_rms(rows, C, 1, 0, 0, C, C, 1e-6)
        mb.bevmap_rms_norm(n, x.data_ptr(), 0, w.data_ptr(), 0, at[4], 0)
        torch.cuda.synchronize()
        ref = [*reversed(bev.rms_norm_add(x, r, w)), bev.rms_norm_int8(x, w)[0], None,
               bev.rms_norm(x, w, out_dtype=torch.float32)]
        for t, expect in zip(out, ref):
            assert (t[:17] == 7).all() and (t[17 + rows * C:] == 7).all(), (rows, C)
            assert expect is None or torch.equal(t[17:17 + rows * C].view(rows, C), expect), (rows, C)
    for rows, F in ((9, 3), (21, 65), (5, 331)):
        x, dy = normal(rows, 2 * F).half(), normal(rows, F).half()
        y, dx = (torch.full((rows * n + 64,), 7.0, device="cuda", dtype=torch.float16) for n in (F, 2 * F))
        held = torch.full((rows * 2 * F + 64,), 7, device="cuda", dtype=torch.int8)
        e = torch.full((rows * 2 * -(-F // 32) + 64,), 7, device="cuda", dtype=torch.uint8)
        g = mb.bevmap_gate(rows, F, 2, 2, 2 * F)
        mb.bevmap_gated_act(g, x.data_ptr(), y.data_ptr() + 34, held.data_ptr() + 17, e.data_ptr() + 17)
        mb.bevmap_gated_act_backward(g, dy.data_ptr(), 0, held.data_ptr() + 17, e.data_ptr() + 17, dx.data_ptr() + 34)
        torch.cuda.synchronize()
        leaf = x.clone().requires_grad_()
        ref = bev.gated_act(leaf, "silu", "int8")
        grad, = torch.autograd.grad(ref, leaf, dy)
        for t, n, expect in ((y, F, ref), (dx, 2 * F, grad), (held, 2 * F, None), (e, 2 * -(-F // 32), None)):
            assert (t[:17] == 7).all() and (t[17 + rows * n:] == 7).all(), (rows, F)
            assert expect is None or torch.equal(t[17:17 + rows * n].view(rows, n), expect), (rows, F)
    for tokens, H, D, P, mixed in ((5, 3, 31, 15, 0), (5, 3, 31, 15, 1), (7, 1, 84, 42, 0), (7, 2, 9, 4, 1), (7, 2, 9, 4, 0),
                                   (3, 3, 45, 20, 0)):
        x = normal(1, tokens, H, D).bfloat16()
        f, place = bev.rotary_frequencies(P, device="cuda"), torch.arange(tokens, device="cuda")[None]
        out = torch.full((x.numel() + 64,), 7.0, device="cuda", dtype=torch.bfloat16)
        mb.bevmap_rotary(mb.bevmap_turn(1, tokens, H, D, P, 1, mixed, 1, 1, 1.0, 0, H * D, D), x.data_ptr(),
                         place.data_ptr(), f.data_ptr(), out.data_ptr() + 34, False)
        torch.cuda.synchronize()
        assert (out[:17] == 7).all() and (out[17 + x.numel():] == 7).all(), (D, P)
        assert torch.equal(out[17:17 + x.numel()].view_as(x), bev.rotary(x, place, f, bool(mixed))), (D, P)


# ---------------------------------------------------------------- rotary positions

def _rotary_reference(torch, x, positions, frequencies, interleaved, amplitude, backward=False):
    x, P = x.double(), frequencies.numel()
    place = positions.double()
    if place.dim() == 2:
        place = place[..., None]
    axis = torch.arange(P, device="cuda") // (P // place.shape[2])
    angle = (place[..., axis] * frequencies)[:, :, None]
    cos, sin = amplitude * angle.cos(), amplitude * angle.sin() * (-1 if backward else 1)
    p = torch.arange(P, device="cuda")
    first, second = (2 * p, 2 * p + 1) if interleaved else (p, p + P)
    a, b = x[..., first], x[..., second]
    y, tol = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    # the fraction of a turn is rounded once, its series ends below 2^-25 and is rounded four times, and two
    # more follow with the amplitude; then two products and a sum
    size = abs(amplitude) * 12 * U32 * (a.abs() + b.abs())
    tol[..., first], tol[..., second] = size, size
    return y, tol


ROTARY_CASES = [
    # batch, tokens, heads, dim, pairs, axes, interleaved, positions, type, packed
    (1, 1, 1, 2, 1, 1, False, "i32", "f32", False),
    (8, 1, 10, 64, 32, 1, False, "i64", "bf16", False),
    (1, 500, 4, 32, 16, 2, False, "f32", "bf16", True),
    (2, 77, 3, 128, 32, 1, True, "i32", "f16", False),
    (2, 77, 3, 128, 32, 1, False, "i32", "f16", True),
    (3, 41, 5, 20, 9, 3, False, "f32", "f32", True),
    (3, 41, 5, 21, 9, 3, True, "i64", "bf16", False),
    (1, 130, 2, 84, 42, 2, True, "f32", "f16", False),
    (1, 130, 2, 84, 42, 1, False, "f32", "f16", False),
    (1, 300, 1, 6, 3, 1, True, "i32", "f32", False),
    (1, 4000, 16, 128, 64, 1, False, "i32", "f32", False),
    (2, 3, 2, 4096, 2048, 1, False, "i64", "bf16", False),
    (2, 3, 2, 4095, 2047, 1, True, "i64", "f32", False),
    (70000, 1, 1, 16, 4, 1, False, "i64", "bf16", True),
]


@pytest.mark.parametrize("batch,tokens,heads,dim,pairs,axes,interleaved,kind,dtype,packed", ROTARY_CASES)
def test_rotary(torch, bev, batch, tokens, heads, dim, pairs, axes, interleaved, kind, dtype, packed):
    normal = _normal(torch, 1)
    to = _dtype(torch, dtype)
    x = (normal(batch, tokens, 2, heads, dim).to(to)[:, :, 1] if packed else normal(batch, tokens, heads, dim).to(to))
    x.requires_grad_()
    gen = torch.Generator(device="cuda").manual_seed(2)
    shape = (batch, tokens) if axes == 1 else (batch, tokens, axes)
    if kind == "f32":
        positions = 100 * torch.rand(shape, generator=gen, device="cuda") - 50
    else:
        positions = torch.randint(-5, 1 << 20, shape, generator=gen, device="cuda",
                                  dtype=torch.int32 if kind == "i32" else torch.int64)
    frequencies = bev.rotary_frequencies(pairs, axes=axes, device="cuda")
    dy = normal(batch, tokens, heads, dim).to(to)
    for amplitude in (1.0, 1.3):
        y = bev.rotary(x, positions, frequencies, interleaved, amplitude)
        dx, = torch.autograd.grad(y, x, dy)
        for what, got, src, backward in (("y", y.detach(), x.detach(), False), ("dx", dx, dy, True)):
            ref, tol = _rotary_reference(torch, src, positions, frequencies, interleaved, amplitude, backward)
            assert got.is_contiguous()
            _check(what, got, ref, tol + 1.01 * _u(dtype) * ref.abs() + _tiny(dtype))
            assert torch.equal(got[..., 2 * pairs:], src[..., 2 * pairs:])


def test_rotary_far_positions(torch, bev):
    """Against angles reduced in exact integer arithmetic."""
    pi = 31415926535897932384626433832795028841971693993751058209749445923       # times 10^64
    positions = torch.tensor([[0, 1, -1, 12345, 10 ** 6, 2 ** 31, -2 ** 40 - 1, 2 ** 53 - 1]], device="cuda")
    frequencies = bev.rotary_frequencies(8, device="cuda")
    x = torch.zeros(1, 8, 1, 16, device="cuda")
    x[..., :8] = 1.0
    y = bev.rotary(x, positions, frequencies)[0, :, 0].double().cpu()
    for i, place in enumerate(positions[0].tolist()):
        for p, f in enumerate(frequencies.tolist()):
            top, bottom = f.as_integer_ratio()
            angle = (place * top * 10 ** 64 // bottom) % (2 * pi) / 10 ** 64
            assert abs(y[i, p].item() - math.cos(angle)) <= 12 * U32, (place, f)
            assert abs(y[i, 8 + p].item() - math.sin(angle)) <= 12 * U32, (place, f)


def test_rotary_views_and_positions_that_are_not_finite(torch, bev):
    normal = _normal(torch, 3)
    x = normal(2, 5, 4, 8)
    f = bev.rotary_frequencies(4, device="cuda")
    place = torch.arange(10, dtype=torch.float32, device="cuda").view(2, 5)
    y = bev.rotary(x, place, f)
    assert torch.equal(bev.rotary(x.transpose(1, 2).contiguous().transpose(1, 2), place, f), y)
    wide = torch.zeros(2, 5, 4, 9, device="cuda")
    wide[..., 1:] = x
    assert torch.equal(bev.rotary(wide[..., 1:], place, f), y)
    shared = x[:, :, :1].expand(-1, -1, 4, -1)
    assert torch.equal(bev.rotary(shared, place, f), bev.rotary(shared.contiguous(), place, f))
    assert torch.equal(bev.rotary(x, place[..., None].contiguous(), f), y)
    assert torch.equal(bev.rotary(x, place.long(), f), y) and torch.equal(bev.rotary(x, place.int(), f), y)
    place[1, 2] = math.inf
    z = bev.rotary(x, place, f)
    assert z[1, 2].isnan().all() and torch.equal(z[0], y[0]) and torch.equal(z[1, 3:], y[1, 3:])
    assert bev.rotary(x[:, :0], place[:, :0].contiguous(), f).shape == (2, 0, 4, 8)


# ---------------------------------------------------------------- gated activation

def _act_reference(torch, g, act):
    """act(g), its slope, and the bounds of both: an exponential or erf of a few roundings, whose
    argument, up to g^2 / 2, is rounded."""
    phi, cdf = torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi), 0.5 * torch.erfc(-g / math.sqrt(2))
    sig = torch.sigmoid(g)
    a, slope = {"none": (g, torch.ones_like(g)), "relu": (g.clamp(min=0), (g > 0).double()),
                "silu": (g * sig, sig * (1 + g * (1 - sig))), "gelu": (g * cdf, cdf + g * phi)}[act]
    own = 8 * U32 * (1 + g.abs()) if act in ("silu", "gelu") else 0 * g
    return a, slope, own * g.abs().clamp(max=1) + 2 * U32 * a.abs(), own * (1 + g.abs()) + 2 * U32 * slope.abs()


def _two_to(torch, e):
    """2^e in 64 bits, from its bits."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _held_reference(torch, x, F):
    """x as integers and exponents of blocks of 32 channels of each half, in 64 bits."""
    t = torch.nn.functional.pad(x.double().reshape(-1, 2, F), (0, -F % 32)).view(-1, 2, -(-F // 32), 32)
    top = t.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(top)
    e = torch.where(top > 0, power - 7 + (part > 127 / 128), -127).clamp(min=-127)
    return torch.round(t * _two_to(torch, -e)).view(-1, 2, t.shape[2] * 32)[..., :F].to(torch.int8), (e + 127).squeeze(-1).to(torch.uint8)


def _value_of(torch, held, exponents):
    F = held.shape[-1]
    return held.double() * _two_to(torch, exponents.long().repeat_interleave(32, -1)[..., :F] - 127)


GATE_CASES = [
    # shape without the halves, columns left of a slice, act, type
    ((1, 1), 0, "silu", "f32"),
    ((1, 320), 0, "silu", "bf16"),
    ((5, 7, 32), 0, "gelu", "f16"),
    ((33, 31), 0, "silu", "f32"),
    ((33, 65), 3, "gelu", "bf16"),
    ((100, 66), 2, "relu", "f16"),
    ((600, 1024), 0, "gelu", "f32"),
    ((1000, 320), 8, "silu", "bf16"),
    ((1000, 328), 0, "none", "bf16"),
    ((77, 4100), 0, "silu", "f16"),
    ((3, 20000), 4, "relu", "f32"),
]


@pytest.mark.parametrize("checkpoint", [None, "int8"])
@pytest.mark.parametrize("shape,left,act,dtype", GATE_CASES)
def test_gated_act(torch, bev, shape, left, act, dtype, checkpoint):
    normal = _normal(torch, 1)
    F, to = shape[-1], _dtype(torch, dtype)
    x = (normal(*shape[:-1], left + 2 * F) * torch.exp(normal(left + 2 * F, s=0.7))).to(to)[..., left:].requires_grad_()
    dy = normal(*shape).to(to)
    y = bev.gated_act(x, act, checkpoint)
    dx, = torch.autograd.grad(y, x, dy)
    with torch.no_grad():
        assert torch.equal(bev.gated_act(x, act, checkpoint), y)
    flat = x.detach().double().reshape(-1, 2, F)
    a, _, a_tol, _ = _act_reference(torch, flat[:, 0], act)
    ref = a * flat[:, 1]
    _check("y", y.detach().reshape(-1, F), ref,
           a_tol * flat[:, 1].abs() + (U32 + 1.01 * _u(dtype)) * ref.abs() + _tiny(dtype))
    if checkpoint:
        held, exponents = _held_reference(torch, x.detach(), F)
        flat = _value_of(torch, held, exponents)
    a, slope, a_tol, slope_tol = _act_reference(torch, flat[:, 0], act)
    d = dy.double().reshape(-1, F)
    ref = torch.stack((d * flat[:, 1] * slope, d * a), 1)
    tol = torch.stack(((d * flat[:, 1]).abs() * slope_tol, d.abs() * a_tol), 1)
    _check("dx", dx.reshape(-1, 2, F), ref, tol + (2 * U32 + 1.01 * _u(dtype)) * ref.abs() + _tiny(dtype))


@pytest.mark.parametrize("features,dtype", [(1, "f32"), (31, "bf16"), (32, "f32"), (40, "f16"), (64, "bf16"),
                                            (130, "f32"), (321, "bf16"), (328, "f16")])
def test_checkpoint_in_8_bits(torch, bev, features, dtype):
    """The integers and exponents themselves, blocks of every size, and of infinities and NaN."""
    from paper_2205_13542_amd import layer_ops
    normal = _normal(torch, 2)
    x = (normal(20, 2 * features) * torch.exp(normal(20, 1, s=3.0))).to(_dtype(torch, dtype))
    x[3] = 0
    x[4] = 127.0                    # exactly at the largest integer
    x[5] = 127.5
    x[6, 0], x[6, features] = -math.inf, math.nan
    if dtype != "f16":
        x[7], x[8] = 3e38, 2.0 ** -125
        x[9] = 2.0 ** -130
    with torch.no_grad():
        y, held, exponents = layer_ops._native.gated_act_held(x, 0)
    rest = [i for i in range(20) if i != 6]
    ref, e = _held_reference(torch, x[rest], features)
    assert torch.equal(held[rest], ref) and torch.equal(exponents[rest], e)
    assert (exponents[6, :, 0] == 255).all() and not held[6, :, :32].any()
    if features > 32:
        assert torch.equal(held[6, :, 32:], _held_reference(torch, x[6:7].nan_to_num(0, 0, 0), features)[0][0, :, 32:])
    back = x.clone().requires_grad_()
    dx, = torch.autograd.grad(bev.gated_act(back, "none", "int8"), back, torch.ones_like(y))
    assert dx[6, features:2 * features][:32].isnan().all() and not dx[rest].isnan().any()


def test_checkpoint_frees_the_input(torch, bev):
    x = torch.randn(20000, 1024, device="cuda", dtype=torch.bfloat16).requires_grad_()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = bev.gated_act(x * 1, checkpoint="int8")
    kept = torch.cuda.memory_allocated() - before
    assert kept <= y.numel() * 2 + x.numel() * 33 / 32 + (1 << 20)
    y.sum().backward()


# ---------------------------------------------------------------- all of them

def test_gradients_against_differences(torch, bev):
    """Central differences along random directions, in fp32 with the sums in 64 bits. Values are of
    order 1, so a step of 1/64 truncates at about 1e-4 of the derivative's size and rounds at about
    1e-5 of it."""
    normal = _normal(torch, 1)
    place = torch.arange(22, device="cuda").view(2, 11)
    f = bev.rotary_frequencies(3, device="cuda")
    calls = [
        (lambda x, w: bev.rms_norm(x, w), [normal(30, 12), normal(12)]),
        (lambda x, r, w: torch.cat(bev.rms_norm_add(x, r, w)), [normal(30, 12), normal(30, 12), normal(12)]),
        (lambda x: bev.rotary(x, place, f, True, 1.2), [normal(2, 11, 3, 8)]),
        (lambda x: bev.gated_act(x, "silu"), [normal(20, 18)]),
        (lambda x: bev.gated_act(x, "gelu"), [normal(20, 18)]),
    ]
    for call, inputs in calls:
        weight = normal(*call(*inputs).shape).double()
        leaves = [t.clone().requires_grad_() for t in inputs]
        grads = torch.autograd.grad((call(*leaves).double() * weight).sum(), leaves)
        for i, g in enumerate(grads):
            along = normal(*inputs[i].shape)
            along /= along.norm()
            step = 2.0 ** -6

            def at(s):
                moved = [t + s * along if j == i else t for j, t in enumerate(inputs)]
                return (call(*moved).double() * weight).sum().item()

            # of fourth order, from two central differences
            got = (8 * (at(step) - at(-step)) - (at(2 * step) - at(-2 * step))) / (12 * step)
            want = (g.double() * along.double()).sum().item()
            assert abs(got - want) <= 1e-3 * (abs(want) + g.double().norm().item() / math.sqrt(g.numel())) + 2e-3


def test_second_derivatives_are_refused(torch, bev):
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    place = torch.arange(4, device="cuda")[None]
    f = bev.rotary_frequencies(2, device="cuda")
    for y in (bev.rms_norm(x), bev.rms_norm_add(x, x)[0], bev.rotary(x.view(1, 4, 1, 8), place, f), bev.gated_act(x)):
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad(y.sum(), x, create_graph=True)


def test_offsets_past_32_bits(torch, bev):
    """Rows whose last ones lie more than 2^31 and 2^32 elements into their buffer."""
    rows, stride = 4200, 1 << 20
    buffer = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")
    wide = buffer.view(rows, stride)
    x = _normal(torch, 9)(rows, 64).bfloat16()
    for first in (0, stride - 64):
        view = wide[:, first:first + 64]
        view.copy_(x)
        assert torch.equal(bev.rms_norm(view), bev.rms_norm(x))
        y, total = bev.rms_norm_add(view, view)
        assert torch.equal(y, bev.rms_norm_add(x, x)[0]) and torch.equal(total, x + x)
        assert all(torch.equal(a, b) for a, b in zip(bev.quantize_int8(view), bev.quantize_int8(x)))
        assert torch.equal(bev.gated_act(view), bev.gated_act(x))
        leaf, near = view.detach().requires_grad_(), x.clone().requires_grad_()
        for call in (bev.rms_norm, bev.gated_act):
            got, = torch.autograd.grad(call(leaf).float().sum(), leaf)
            ref, = torch.autograd.grad(call(near).float().sum(), near)
            assert torch.equal(got, ref)
        f = bev.rotary_frequencies(8, device="cuda")
        place = torch.arange(rows, device="cuda")[None]
        assert torch.equal(bev.rotary(view.view(1, rows, 4, 16), place, f),
                           bev.rotary(x.view(1, rows, 4, 16), place, f))
    del buffer, wide, view, leaf
    q = torch.zeros(rows * stride, dtype=torch.int8, device="cuda").view(rows, stride)
    held, scale = bev.quantize_int8(x)
    w, ws = _held(torch, 3, 48, 64)
    q[:, stride - 64:] = held
    assert torch.equal(bev.linear_int8(q[:, stride - 64:], scale, w, ws), bev.linear_int8(held, scale, w, ws))
    q[:, stride - 63:] = held[:, :63]
    assert torch.equal(bev.linear_int8(q[:, stride - 63:], scale, w[:, :63], ws),
                       bev.linear_int8(held[:, :63].contiguous(), scale, w[:, :63].contiguous(), ws))


def test_results_past_32_bits(torch, bev):
    """More than 2^32 elements of result, by a sample of rows."""
    x = _normal(torch, 9)(1 << 16, 64).bfloat16()
    rows = torch.arange(1100000, device="cuda") % (1 << 16)
    held, scale = bev.quantize_int8(x)
    w, ws = _held(torch, 3, 4000, 64)
    y = bev.linear_int8(held[rows], scale[rows], w, ws)
    pick = torch.tensor([0, 1, 524287, 536871, 1073742, 1099998, 1099999], device="cuda")
    assert torch.equal(y[pick], bev.linear_int8(held, scale, w, ws)[rows[pick]])


def _layer_inputs(torch, bev):
    """A decoder layer's leaves: queries, their residual stream, the map's states, weights."""
    normal = _normal(torch, 7)
    leaves = [normal(2, 30, 64).bfloat16(), normal(2, 30, 64).bfloat16(), normal(2, 420, 64).bfloat16(),
              1 + normal(64, s=0.1), normal(64, 64, s=0.125).bfloat16(), normal(64, 128, s=0.125).bfloat16(),
              normal(64, 192, s=0.125).bfloat16(), normal(96, 64, s=0.1).bfloat16()]
    cells = torch.stack((torch.arange(420, device="cuda") % 21, torch.arange(420, device="cuda") // 21), -1)
    places = [cells.float().expand(2, -1, -1).contiguous(),
              20 * torch.rand((2, 30, 2), generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")]
    return leaves, places, bev.rotary_frequencies(8, base=100.0, axes=2, device="cuda"), normal(2, 30, 64).bfloat16()


def _layer(torch, bev, leaves, places, f):
    """One layer of a decoder, from the queries' stream to the stream behind the feed-forward layer."""
    x, stream, states, w, wq, wkv, wup, wdown = leaves
    normed, stream = bev.rms_norm_add(x, stream, w)
    q = bev.rotary((normed @ wq).view(2, 30, 4, 16), places[1], f)
    k, v = (states @ wkv).view(2, 420, 2, 4, 16).unbind(2)
    heard = bev.cross_attention(q, bev.rotary(k, places[0], f), v)
    normed, stream = bev.rms_norm_add(bev.dropout_add(heard.flatten(2), 0.1, 3, 1), stream, w)
    fed = bev.gated_act(normed @ wup, checkpoint="int8") @ wdown
    return fed + stream


def _step(torch, bev, leaves, places, f, dy):
    leaves = [t.detach().requires_grad_() for t in leaves]
    y = _layer(torch, bev, leaves, places, f)
    return [y.detach(), *torch.autograd.grad(y, leaves, dy)]


def test_a_layer_trains(torch, bev):
    """The whole layer's output and gradients against torch's own operations in 64 bits. bf16 is rounded
    to some ten times on the way of a number, each by 2^-9 of its size on average, and the checkpoint adds
    1 / 254 of a block's largest at most: 5% of the norm is several times of that, a mistake is more."""
    leaves, places, f, dy = _layer_inputs(torch, bev)
    got = _step(torch, bev, leaves, places, f, dy)
    # the mask that the dropout drew
    kept = bev.dropout_add(torch.ones(2, 30, 64, device="cuda"), 0.1, 3, 1).double().cpu()
    x, stream, states, w, wq, wkv, wup, wdown = ref = [t.detach().double().cpu().requires_grad_() for t in leaves]

    def norm(t):
        return t / torch.sqrt(t.square().mean(-1, keepdim=True) + 1e-6) * w

    def turn(t, place):
        angle = (place.double().cpu().repeat_interleave(4, -1) * f.cpu())[:, :, None]
        a, b = t.chunk(2, -1)
        return torch.cat((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1)

    h = x + stream
    q = turn((norm(h) @ wq).view(2, 30, 4, 16), places[1]).transpose(1, 2)
    k, v = (states @ wkv).view(2, 420, 2, 4, 16).unbind(2)
    p = torch.softmax(q @ turn(k, places[0]).permute(0, 2, 3, 1) / 4, -1)
    h = h + (p @ v.transpose(1, 2)).transpose(1, 2).flatten(2) * kept
    gate, value = (norm(h) @ wup).chunk(2, -1)
    y = (gate * torch.sigmoid(gate) * value) @ wdown + h
    want = [y.detach(), *torch.autograd.grad(y, ref, dy.double().cpu())]
    for i, (a, b) in enumerate(zip(got, want)):
        assert (a.double().cpu() - b).norm() <= 0.05 * b.norm(), i


def test_a_layer_serves_in_8_bits(torch, bev):
    """Norm, projection and feed-forward layer in 8 bits beside the same in 64: a number held in 8 bits
    is off by at most 1 / 254 of its row's largest, about 1% of its row's root mean square on average; four
    products of such pairs lie between, so 5% of the norm is some times of that."""
    normal = _normal(torch, 4)
    x, stream = normal(5, 256).bfloat16(), normal(5, 256).bfloat16()
    w = 1 + normal(256, s=0.1)
    wide, down = normal(1024, 256, s=1 / 16), normal(256, 512, s=1 / 22)
    up8, down8 = bev.quantize_int8(wide), bev.quantize_int8(down)
    held, scale, total = bev.rms_norm_add_int8(x, stream, w)
    y = bev.linear_int8(held, scale, *up8)
    y = bev.linear_int8(*bev.quantize_int8(bev.gated_act(y)), *down8)
    h = x.double() + stream.double()
    ref = (h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6) * w.double()) @ wide.double().t().contiguous()
    gate, value = ref.chunk(2, 1)
    ref = (gate * torch.sigmoid(gate) * value) @ down.double().t().contiguous()
    assert (y.double() - ref).norm() <= 0.05 * ref.norm()
    one = bev.rms_norm_add_int8(x[2:3], stream[2:3], w)     # a token alone gets what it gets among others
    alone = bev.linear_int8(one[0], one[1], *up8)
    alone = bev.linear_int8(*bev.quantize_int8(bev.gated_act(alone)), *down8)
    assert torch.equal(alone, y[2:3])


def test_a_step_on_another_stream(torch, bev):
    """Forward and backward on a side stream, on inputs made there, with nothing else to order them."""
    leaves, places, f, dy = _layer_inputs(torch, bev)
    ref = _step(torch, bev, leaves, places, f, dy)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        mine, there = [torch.empty_like(t) for t in leaves], [torch.empty_like(t) for t in places]
        grad, turns = torch.empty_like(dy), torch.empty_like(f)
        big = torch.randn(1 << 26, device="cuda")
        for _ in range(8):
            big = big * 1.5                     # keeps the stream busy
        for t, a in zip((*mine, *there, grad, turns), (*leaves, *places, dy, f)):
            t.copy_(a)
        got = _step(torch, bev, mine, there, turns, grad)
    side.synchronize()
    assert all(torch.equal(a, r) for a, r in zip(got, ref))


def test_a_step_in_a_graph(torch, bev):
    leaves, places, f, dy = _layer_inputs(torch, bev)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _step(torch, bev, leaves, places, f, dy)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(torch, bev, leaves, places, f, dy)
    for i in range(4):
        gen = torch.Generator(device="cuda").manual_seed(60 + i)
        for t in (leaves[0], leaves[2], dy, places[1]):
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
        graph.replay()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        ref = _step(torch, bev, leaves, places, f, dy)
        assert all(torch.equal(a, r) for a, r in zip(got, ref)), f"replay {i}"


def test_serving_in_two_graphs(torch, bev):
    """Two captured graphs of the serving calls, replayed in turn on inputs that change."""
    normal = _normal(torch, 6)
    x, stream, w = normal(3, 512).bfloat16(), normal(3, 512).bfloat16(), 1 + normal(512, s=0.1)
    weights = bev.quantize_int8(normal(700, 512))

    def call():
        held, scale, total = bev.rms_norm_add_int8(x, stream, w)
        return bev.linear_int8(held, scale, *weights), total

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(call())
    for i in range(4):
        x.copy_(normal(3, 512))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        ref = call()
        for out in outs:
            assert all(torch.equal(a, r) for a, r in zip(out, ref)), f"replay {i}"


@pytest.mark.parametrize("rows,channels,features", [(16500, 592, 1000), (16390, 597, 1021), (4096, 80, 2056),
                                                    (3000, 331, 2000), (700, 2000, 777), (60, 400, 400)])
def test_linear_int8_in_a_graph(torch, bev, rows, channels, features):
    """Every size of tile, first called while it is captured."""
    x, xs = _held(torch, 8, rows, channels)
    w, ws = _held(torch, 9, features, channels)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = bev.linear_int8(x, xs, w, ws, out_dtype=torch.float32)
    for i in range(3):
        x.copy_(_held(torch, 10 + i, rows, channels)[0])
        graph.replay()
        assert torch.equal(y, bev.linear_int8(x, xs, w, ws, out_dtype=torch.float32)), f"replay {i}"


def test_empty_inputs(torch, bev):
    x = torch.zeros(0, 8, device="cuda", requires_grad=True)
    w = torch.ones(8, device="cuda", requires_grad=True)
    y, total = bev.rms_norm_add(x, x, w)
    dx, dw = torch.autograd.grad(y.sum() + total.sum(), (x, w))
    assert dx.shape == (0, 8) and dw.shape == (8,) and not dw.any()
    y = bev.gated_act(x, checkpoint="int8")
    assert y.shape == (0, 4) and torch.autograd.grad(y.sum(), x)[0].shape == (0, 8)
    assert bev.rms_norm_int8(x.detach())[0].shape == (0, 8) and bev.quantize_int8(x.detach())[1].shape == (0,)


def test_hooks_on_saved_tensors(torch, bev):
    """Saved tensors that come back with other strides, from the host or another layout, give
    the same gradients; another size or dtype is refused."""
    normal = _normal(torch, 3)
    place = torch.arange(20, device="cuda").view(2, 10)
    f = bev.rotary_frequencies(3, device="cuda")
    w = normal(24)
    packed = normal(20, 3 * 24)
    wide = packed[:, 24:48]                          # rows 72 elements apart
    half = packed.bfloat16()[:, 24:48]

    def spread(t):                                   # each row followed by a row of something else
        if t.dim() != 2:
            return t
        room = torch.full((t.shape[0], 2 * t.shape[1]), 9, dtype=t.dtype, device=t.device)
        room[:, ::2] = t
        return room[:, ::2]

    hooks = [
        lambda: torch.autograd.graph.save_on_cpu(),
        lambda: torch.autograd.graph.saved_tensors_hooks(spread, lambda t: t),
        lambda: torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.clone(memory_format=torch.contiguous_format)),
    ]
    calls = [
        (lambda x, w: bev.rms_norm(x, w), wide),
        (lambda x, w: bev.rms_norm(x, w), half),
        (lambda x, w: torch.cat(bev.rms_norm_add(x, x.detach(), w)), wide),
        (lambda x, w: torch.cat(bev.rms_norm_add(x.detach(), x, w)), half),
        (lambda x, w: bev.gated_act(x) * w[:12], wide),
        (lambda x, w: bev.gated_act(x, "gelu", checkpoint="int8") * w[:12], half),
        (lambda x, w: bev.rotary(x.unflatten(0, (2, 10)).unflatten(-1, (3, 8)), place, f).flatten(-2) * w, wide),
    ]
    for call, x in calls:
        leaf, weight = x.detach().requires_grad_(), w.clone().requires_grad_()
        dy = None
        grads = []
        for hook in [None, *hooks]:
            if hook is None:
                y = call(leaf, weight)
                dy = _normal(torch, 4)(*y.shape).to(y.dtype)
            else:
                with hook():
                    y = call(leaf, weight)
            grads.append(torch.autograd.grad(y, (leaf, weight), dy))
        for other in grads[1:]:
            assert all(torch.equal(a, b) for a, b in zip(grads[0], other))

    def changes(t):
        return t[..., :1].clone() if t.dtype != torch.float64 else t.float()

    for call, x in (*calls[:4], *((lambda x, w, c=c: c(x, torch.ones_like(w.detach())), x) for c, x in calls[4:])):
        leaf = x.detach().requires_grad_()
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, changes):
            y = call(leaf, w)
            with pytest.raises(RuntimeError):
                torch.autograd.grad(y.float().sum(), leaf)


def test_views_that_negate(torch, bev):
    """A view that negates what lies in memory is refused as an input and resolved as a gradient."""
    x, dy = _normal(torch, 1)(6, 16), _normal(torch, 2)(6, 16)
    place, f = torch.arange(6, device="cuda")[None], bev.rotary_frequencies(4, device="cuda")
    calls = [bev.rms_norm, lambda t: bev.rms_norm_add(t, t)[1],
             lambda t: bev.gated_act(torch.cat((t, t), -1), checkpoint="int8"),
             lambda t: bev.rotary(t.view(1, 6, 1, 16), place, f).view(6, 16)]
    for call in calls:
        leaf = x.clone().requires_grad_()
        got, = torch.autograd.grad(call(leaf), leaf, torch._neg_view(dy))
        ref, = torch.autograd.grad(call(leaf), leaf, -dy)
        assert torch.equal(got, ref)
    for call in (bev.rms_norm, bev.quantize_int8, bev.gated_act,
                 lambda t: bev.rotary(t.view(1, 6, 1, 16), place, f), lambda t: bev.rms_norm(x, t[0])):
        with pytest.raises(bev.BevpoolError, match="resolve_neg"):
            call(torch._neg_view(x))


def test_refusals(torch, bev):
    x = torch.zeros(6, 5, 8, device="cuda")
    q, s = torch.zeros(6, 8, dtype=torch.int8, device="cuda"), torch.ones(6, device="cuda")
    t = torch.zeros(2, 3, 4, 8, device="cuda")
    place, f = torch.zeros(2, 3, device="cuda"), bev.rotary_frequencies(4, device="cuda")
    leaf = x.clone().requires_grad_()
    bad = [
        lambda: bev.rms_norm(x.double()),
        lambda: bev.rms_norm(x, torch.ones(7, device="cuda")),
        lambda: bev.rms_norm(x, torch.ones(8)),
        lambda: bev.rms_norm(x, out_dtype=torch.int8),
        lambda: bev.rms_norm(x, eps=-1.0),
        lambda: bev.rms_norm(x, eps=math.nan),
        lambda: bev.rms_norm(x.transpose(0, 2)),
        lambda: bev.rms_norm(x[:, ::2]),
        lambda: bev.rms_norm(torch.zeros(2, 8193, device="cuda")),
        lambda: bev.rms_norm(torch.zeros(2, 0, device="cuda")),
        lambda: bev.rms_norm(torch.zeros((), device="cuda")),
        lambda: bev.rms_norm_add(x, x[:5]),
        lambda: bev.rms_norm_add(x, x.half()),
        lambda: bev.rms_norm_add(x, x.cpu()),
        lambda: bev.rms_norm_int8(leaf),
        lambda: bev.rms_norm_add_int8(x, leaf),
        lambda: bev.rms_norm_int8(x, torch.ones(8, device="cuda", requires_grad=True)),
        lambda: bev.quantize_int8(leaf),
        lambda: bev.quantize_int8(q),
        lambda: bev.quantize_int8(torch.zeros(1, 131072, device="cuda")),
        lambda: bev.linear_int8(q, s, q.float(), s),
        lambda: bev.linear_int8(q.float(), s, q, s),
        lambda: bev.linear_int8(q, s, q[:, :7], s),
        lambda: bev.linear_int8(q, s, q[0], s),
        lambda: bev.linear_int8(q, s[:5], q, s),
        lambda: bev.linear_int8(q, s, q, s[:5]),
        lambda: bev.linear_int8(q, s.half(), q, s),
        lambda: bev.linear_int8(q, s, q, s, bias=s.bfloat16()),
        lambda: bev.linear_int8(q, s, q, s, bias=s[:5]),
        lambda: bev.linear_int8(q, s, q, s, out_dtype=torch.int32),
        lambda: bev.linear_int8(q.t(), s[:1].expand(8), q, s),
        lambda: bev.linear_int8(q, s.clone().requires_grad_(), q, s),
        lambda: bev.linear_int8(torch.zeros(1, 131072, dtype=torch.int8, device="cuda"), s[:1],
                                torch.zeros(1, 131072, dtype=torch.int8, device="cuda"), s[:1]),
        lambda: bev.rotary(t[0], place, f),
        lambda: bev.rotary(t.double(), place, f),
        lambda: bev.rotary(t, place[:1], f),
        lambda: bev.rotary(t, place.double(), f),
        lambda: bev.rotary(t, place, f.float()),
        lambda: bev.rotary(t, place, bev.rotary_frequencies(5, device="cuda")),
        lambda: bev.rotary(t, place, f[:0]),
        lambda: bev.rotary(t, torch.zeros(2, 3, 3, device="cuda"), f),
        lambda: bev.rotary(t, torch.zeros(2, 3, 0, device="cuda"), f),
        lambda: bev.rotary(t, place, f, amplitude=math.inf),
        lambda: bev.rotary(t.transpose(2, 3), place, f[:2]),
        lambda: bev.rotary(t, place.t().contiguous().t(), f),
        lambda: bev.rotary(t, place, f.clone().requires_grad_()),
        lambda: bev.rotary(t, place.clone().requires_grad_(), f),
        lambda: bev.rotary(torch.zeros(1, 1, 1, 4098, device="cuda"), place[:1, :1], f),
        lambda: bev.gated_act(x[..., :7]),
        lambda: bev.gated_act(x, act="tanh"),
        lambda: bev.gated_act(x, checkpoint="int4"),
        lambda: bev.gated_act(x.double()),
        lambda: bev.gated_act(x.transpose(0, 2)),
        lambda: bev.gated_act(x[..., :0]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(bev.BevpoolError):
            call()
            print(f"call {i} was not refused", flush=True)
    with torch.no_grad():       # where no gradient is asked for
        bev.rms_norm_int8(leaf), bev.quantize_int8(leaf)
