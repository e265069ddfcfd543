"""GPU tests of layers in the clear against their formulas in 64 bits on the CPU.

Tolerances, with u = 2^-24 (half a step of f32, relative to the value):
  product   f32 steps are the conversion of the sum, two scales and the bias: 3u of the product and u of the result, then half a
            step of the output's type; whole numbers are equal.
  8 bits    a value y of a row carries an error e(y) from its own f32 steps (named at each test).  scale = max|y| / 127 is off by at most
            max e / 127 and two roundings; q is y / scale, off by half a step and by what the errors of y and of the scale move it."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FLOATS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WHOLE = {"i32": torch.int32, "sign": torch.int8, "bits": torch.uint8}


@pytest.fixture(scope="module")
def T():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    import paper_1806_03461_amd
    return paper_1806_03461_amd


def rng(seed):
    return torch.Generator().manual_seed(seed)


def int8(g, m, k, low=-128):
    return torch.randint(low, 128, (m, k), generator=g, dtype=torch.int8)


def strided(t, pad, lead=0):
    """t on the GPU as rows `pad` values further apart than they are long, the first one `lead` values behind an aligned address."""
    m, k = t.shape
    flat = torch.full((lead + m * (k + pad) + 1,), 77, dtype=t.dtype, device="cuda")
    v = flat[lead:lead + m * (k + pad)].view(m, k + pad)[:, :k]
    v.copy_(t)
    return v


# ---- the product -----------------------------------------------------------------------------------------------------

def check_product(T, x, w, out_type, scales=True, bias=True, pads=(0, 0, 0), leads=(0, 0, 0), seed=0):
    g = rng(seed + 1000)
    m, k = x.shape
    n = w.shape[0]
    whole = out_type in WHOLE
    sx = torch.exp(torch.randn(m, generator=g)) if scales and not whole else None
    sw = 0.01 * torch.exp(torch.randn(n, generator=g)) if scales and not whole else None
    b = None
    if bias:
        b = torch.randint(-300, 300, (n,), generator=g, dtype=torch.int32) if whole else torch.randn(n, generator=g)
    dtype = WHOLE[out_type] if whole else FLOATS[out_type]
    out = strided(torch.full((m, n), 55).to(dtype), pads[2], leads[2])
    base = out._base if out._base is not None else out
    before = base.clone()
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    T.bnn_dense_clear(strided(x, pads[0], leads[0]), strided(w, pads[1], leads[1]), out, x_scale=dev(sx), w_scale=dev(sw), bias=dev(b))
    got, after = out.cpu(), base.clone()
    acc = x.double() @ w.double().t()
    if whole:
        acc = acc + (0 if b is None else b.double())
        want = {"i32": acc, "sign": torch.where(acc >= 0, 1.0, -1.0), "bits": (acc >= 0).double()}[out_type]
        assert torch.equal(got.double(), want)
    else:
        y = acc * (1 if sx is None else sx.double()[:, None]) * (1 if sw is None else sw.double())
        want = y if b is None else y + b.double()
        half = torch.finfo(dtype).eps / 2
        bound = 3 * U * y.abs() * (1 + 1e-6) + (U + half) * want.abs() * (1 + 2 * half) + torch.finfo(dtype).smallest_normal * half
        fits = want.abs() < torch.finfo(dtype).max * 0.99
        assert bool(((got.double() - want).abs() <= bound)[fits].all()), float(((got.double() - want).abs() / bound)[fits].max())
    out.copy_(torch.full((m, n), 55).to(dtype))    # what lies between and behind the rows is as it was
    assert torch.equal(base, before) and after.shape == before.shape
    mask = torch.ones_like(base, dtype=torch.bool)
    torch.as_strided(mask, out.shape, out.stride(), out.storage_offset()).fill_(False)
    assert torch.equal(after[mask], before[mask])
    return got


SHAPES = [(1, 1, 1), (1, 16, 4096), (1, 257, 90), (2, 31, 63), (3, 64, 64), (5, 33, 65), (8, 512, 784), (15, 17, 127), (16, 48, 128),
          (17, 100, 129), (31, 256, 255), (32, 1000, 1704), (33, 65, 1705), (48, 128, 4097), (63, 130, 192), (64, 512, 784), (65, 10, 256),
          (127, 255, 513), (128, 128, 1024), (129, 257, 1001), (200, 1111, 2050), (255, 300, 640), (256, 256, 256), (257, 513, 127), (333, 700, 385),
          (512, 1024, 512), (700, 64, 96), (1025, 769, 320)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("out", ["f32", "i32"])
def test_product_shapes(T, shape, out):
    m, n, k = shape
    g = rng(m * 7 + n * 3 + k)
    check_product(T, int8(g, m, k), int8(g, n, k), out, seed=k)


@pytest.mark.parametrize("out", ["f32", "bf16", "f16", "i32", "sign", "bits"])
@pytest.mark.parametrize("m", [1, 7, 40, 150, 300])
def test_product_outputs(T, m, out):
    g = rng(m)
    for bias in (True, False):
        check_product(T, int8(g, m, 200), int8(g, 77, 200), out, bias=bias, seed=m)
        check_product(T, int8(g, m, 256), int8(g, 128, 256), out, bias=bias, scales=False, seed=m)


@pytest.mark.parametrize("pads, leads", [((1, 3, 5), (0, 0, 0)), ((16, 32, 4), (16, 0, 2)), ((0, 0, 0), (1, 2, 1)), ((7, 0, 1), (3, 16, 3)),
                                         ((128, 128, 128), (0, 0, 0)), ((4, 8, 2), (4, 8, 0))])
@pytest.mark.parametrize("shape", [(1, 130, 513), (1, 512, 1024), (13, 70, 256), (40, 96, 1024), (70, 257, 100), (300, 260, 384), (520, 516, 272)],
                         ids=lambda s: "x".join(map(str, s)))
def test_product_strides_and_alignment(T, shape, pads, leads):
    m, n, k = shape
    g = rng(m + n + k)
    for out in ("bf16", "f32", "sign", "i32"):
        check_product(T, int8(g, m, k), int8(g, n, k), out, pads=pads, leads=leads, seed=n)


KS = [4, 60, 64, 68, 128, 132, 192, 200, 256, 260, 320, 384, 392, 448, 452, 512, 576, 580, 640, 708, 768, 896, 1028, 1152, 1292]


@pytest.mark.parametrize("m, n", [(11, 9001), (29, 300), (29, 5003), (97, 161), (4105, 69), (4625, 1665), (3285, 587), (898, 4435), (4663, 2562)])
@pytest.mark.parametrize("more", [0, 1, 2, 12])
def test_product_of_every_number_of_steps(T, m, n, more):
    """Sizes at which each way to split the outputs is the one taken, none of them a whole number of its tiles, with k of none to twenty steps, whole and
    not; rows at multiples of 4 and 16 bytes and at any address.  The sums are whole numbers below 2^53, which a product in 64 bits has exactly."""
    g = torch.Generator(device="cuda").manual_seed(m + more)
    for k in KS:
        k += more
        x, w = (torch.randint(-128, 128, (r, k), generator=g, device="cuda", dtype=torch.int8) for r in (m, n))
        wide = torch.full((m + 1, n + 3), -7, dtype=torch.int32, device="cuda")
        T.bnn_dense_clear(x, w, wide[:m, :n])
        want = x.double() @ w.double().t()
        assert torch.equal(wide[:m, :n].double(), want), k
        assert bool((wide[m] == -7).all()) and bool((wide[:, n:] == -7).all()), k
        if k % 64 < 8:
            sx, sw, b = torch.rand(m, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
            out = torch.empty(m, n, dtype=torch.float16, device="cuda")
            T.bnn_dense_clear(x, w, out, x_scale=sx, w_scale=sw * 1e-3, bias=b)
            y = want * sx.double()[:, None] * (sw * 1e-3).double()
            full = y + b.double()
            bound = 3 * U * y.abs() * (1 + 1e-6) + (U + 2.0 ** -11) * full.abs() * (1 + 2.0 ** -10) + 2.0 ** -25
            assert bool(((out.double() - full).abs() <= bound).all()), k


@pytest.mark.parametrize("m, n", [(1, 5), (20, 40), (100, 130), (300, 520)])
def test_product_of_extremes(T, m, n):
    """-128 times -128 over the longest rows: the sum's last place before 2^31; and rows of all kinds of ends."""
    k = 131071
    x, w = torch.full((m, k), -128, dtype=torch.int8), torch.full((n, k), -128, dtype=torch.int8)
    w[::2] = 127
    out = torch.empty(m, n, dtype=torch.int32, device="cuda")
    T.bnn_dense_clear(x.cuda(), w.cuda(), out)
    row = torch.where(torch.arange(n) % 2 == 0, -128 * 127 * k, 128 * 128 * k).to(torch.int32)
    assert torch.equal(out.cpu(), row.expand(m, n))
    big = torch.full((n,), 2**31 - 1, dtype=torch.int32, device="cuda")     # the sign does not overflow, the sum wraps
    sign = torch.empty(m, n, dtype=torch.int8, device="cuda")
    T.bnn_dense_clear(x.cuda(), w.cuda(), sign, bias=big)
    assert bool((sign == 1).all())
    T.bnn_dense_clear(x.cuda(), w.cuda(), out, bias=big)
    assert torch.equal(out.cpu().long(), ((row.long() + 2**31 - 1 + 2**31) % 2**32 - 2**31).expand(m, n))


def test_product_without_terms_and_without_channels(T):
    x, w = torch.empty(3, 0, dtype=torch.int8, device="cuda"), torch.empty(5, 0, dtype=torch.int8, device="cuda")
    b = torch.randn(5, device="cuda")
    out = torch.full((3, 5), 9.0, device="cuda")
    T.bnn_dense_clear(x, w, out, bias=b)
    assert torch.equal(out, b.expand(3, 5))
    sign = torch.full((3, 5), 9, dtype=torch.int8, device="cuda")
    T.bnn_dense_clear(x, w, sign)
    assert bool((sign == 1).all())
    T.bnn_dense_clear(torch.empty(0, 8, dtype=torch.int8, device="cuda"), torch.empty(5, 8, dtype=torch.int8, device="cuda"),
                      torch.empty(0, 5, device="cuda"))
    T.bnn_dense_clear(torch.empty(3, 8, dtype=torch.int8, device="cuda"), torch.empty(0, 8, dtype=torch.int8, device="cuda"),
                      torch.empty(3, 0, device="cuda"))


def test_product_scales_that_are_not_finite_stay_so(T):
    g = rng(3)
    x, w = int8(g, 4, 64), int8(g, 8, 64)
    x[1] = 0
    sx = torch.tensor([1.0, math.inf, math.nan, 0.0])
    out = torch.empty(4, 8, device="cuda")
    T.bnn_dense_clear(x.cuda(), w.cuda(), out, x_scale=sx.cuda())
    got = out.cpu()
    assert bool(torch.isfinite(got[0]).all()) and bool(torch.isnan(got[1:3]).all()) and bool((got[3] == 0).all())


def test_product_beyond_32_bits_of_offset(T):
    """Rows 2^31 - 64 bytes apart: the third begins behind 2^32."""
    ld, k = 2**31 - 64, 96
    flat = torch.zeros(2 * ld + 4096, dtype=torch.int8, device="cuda")
    x = torch.as_strided(flat, (3, k), (ld, 1))
    g = rng(9)
    hx, hw = int8(g, 3, k), int8(g, 20, k)
    x.copy_(hx)
    out = torch.empty(3, 20, dtype=torch.int32, device="cuda")
    T.bnn_dense_clear(x, hw.cuda(), out)
    assert torch.equal(out.cpu(), (hx.int() @ hw.int().t()))
    out = torch.empty(20, 3, dtype=torch.int32, device="cuda")
    T.bnn_dense_clear(hw.cuda(), x, out)
    assert torch.equal(out.cpu(), (hw.int() @ hx.int().t()))


def test_product_of_rows_far_apart(T):
    """The widest strides that go straight to LDS, 4 MiB, and one beyond: a tile's rows span a gigabyte.  Largest tiles, ragged."""
    m, n, k = 4663, 2562, 132
    for ld in (2 ** 22, 2 ** 22 + 4):
        g = torch.Generator(device="cuda").manual_seed(ld)
        hx, hw = (torch.randint(-128, 128, (r, k), generator=g, device="cuda", dtype=torch.int8) for r in (m, n))
        x, w = (torch.as_strided(torch.empty(ld * r, dtype=torch.int8, device="cuda"), (r, k), (ld, 1)) for r in (m, n))
        x.copy_(hx)
        w.copy_(hw)
        out = torch.empty(m, n, dtype=torch.int32, device="cuda")
        T.bnn_dense_clear(x, w, out)
        assert torch.equal(out.double(), hx.double() @ hw.double().t())
        del x, w
    torch.cuda.empty_cache()


def test_one_tensor_in_two_places(T):
    """The same tensor as both operands of the product, as x and residual (and total), as gate and up."""
    g = rng(6)
    x = int8(g, 70, 200)
    d, out = x.cuda(), torch.empty(70, 70, dtype=torch.int32, device="cuda")
    T.bnn_dense_clear(d, d, out)
    assert torch.equal(out.cpu(), x.int() @ x.int().t())
    f = values(g, 7, 1500, torch.bfloat16)
    q, scale, q2, scale2 = (torch.empty(7, 1500, dtype=torch.int8, device="cuda"), torch.empty(7, device="cuda"),
                            torch.empty(7, 1500, dtype=torch.int8, device="cuda"), torch.empty(7, device="cuda"))
    a, b = f.cuda(), f.cuda()
    T.bnn_rms_norm_clear(a, None, 1e-5, q, scale, residual=a, total=a)
    T.bnn_rms_norm_clear(b, None, 1e-5, q2, scale2, residual=f.cuda())
    assert torch.equal(q, q2) and torch.equal(scale, scale2) and torch.equal(a.cpu(), 2 * f)
    T.bnn_gate_clear(b, b, "silu", q, scale)
    T.bnn_gate_clear(b, f.cuda(), "silu", q2, scale2)
    assert torch.equal(q, q2) and torch.equal(scale, scale2)


@pytest.mark.parametrize("m, n", [(68_000_000, 1), (3, 17_000_000)])
def test_product_of_more_tiles_than_a_launch_takes(T, m, n):
    x = (torch.arange(m, device="cuda") % 251 - 125).to(torch.int8)[:, None]
    w = (torch.arange(n, device="cuda") % 241 - 120).to(torch.int8)[:, None]
    out = torch.empty(m, n, dtype=torch.int32, device="cuda")
    T.bnn_dense_clear(x, w, out)
    assert torch.equal(out, x.int() * w.int().t())


# ---- rows to 8 bits --------------------------------------------------------------------------------------------------

def check_8bit(y, e, q, scale):
    """y in 64 bits, e: how far an f32 evaluation may be from it, value by value."""
    top = y.abs().amax(dim=1)
    floor = 2.0 ** -149
    want = top / 127
    worst = e.amax(dim=1)
    off = (scale.double() - want).abs()
    assert bool((off <= (worst / 127 + 2 * U * want) * (1 + 1e-5) + floor).all()), float((off / (want + floor)).max())
    live = want > 0
    real = torch.zeros_like(y)
    real[live] = y[live] / want[live][:, None]
    slack = torch.zeros_like(y)
    slack[live] = e[live] / want[live][:, None] + real[live].abs() * (worst[live] / top[live])[:, None] + 127 * 2 * U
    far = (q.double() - real).abs()
    assert bool((far <= 0.5 + 1.01 * slack).all()), float((far - 0.5 - slack).max())
    assert int(q.min()) >= -127


def check_norm(T, x, residual=None, weight=None, eps=1e-5, total=True, pad=0, lead=0, in_place=None):
    m, k = x.shape
    dx = strided(x, pad, lead)
    dr = None if residual is None else strided(residual, 2 * pad, lead)
    dt = {"x": dx, "residual": dr, None: strided(torch.zeros_like(x), 3 * pad, lead) if total else None}[in_place]
    q = strided(torch.full((m, k), 33, dtype=torch.int8), pad, 3 * lead)
    scale = torch.full((m,), -1.0, device="cuda")
    T.bnn_rms_norm_clear(dx, None if weight is None else weight.cuda(), eps, q, scale, residual=dr, total=dt)
    h = x.double() + (0 if residual is None else residual.double())
    if dt is not None:
        # f32 rounding of the sum, then the type's; a number of the type itself is met exactly without a residual
        half = torch.finfo(x.dtype).eps / 2
        assert bool(((dt.cpu().double() - h).abs() <= (half + U) * h.abs() + torch.finfo(x.dtype).smallest_normal * half).all())
        if residual is None:
            assert torch.equal(dt.cpu(), x)
    y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps) * (1 if weight is None else weight.double())
    # h one rounding, times weight another, and the mean of squares carries the roundings of h
    check_8bit(y, 3 * U * y.abs(), q.cpu(), scale.cpu())
    if pad:
        between = q._base.clone()
        torch.as_strided(between, q.shape, q.stride(), q.storage_offset()).fill_(77)
        assert bool((between == 77).all())


def values(g, m, k, dtype):
    v = torch.randn(m, k, generator=g) * torch.where(torch.rand(k, generator=g) < 0.02, 10.0, 1.0)
    return v.to(dtype)


LENGTHS = [1, 2, 7, 8, 9, 63, 64, 90, 511, 512, 513, 784, 1001, 1024, 1704, 2048, 2049, 4096, 4100, 8192, 8193, 10240, 16384, 16385, 30001, 32768, 65535, 65536]


@pytest.mark.parametrize("name", FLOATS)
@pytest.mark.parametrize("k", [k for k in LENGTHS if k <= 32768])
def test_norm_lengths(T, k, name):
    g = rng(k)
    t = FLOATS[name]
    for m in (1, 6):
        check_norm(T, values(g, m, k, t), values(g, m, k, t), (1 + 0.2 * torch.randn(k, generator=g)).to(t))
    check_norm(T, values(g, 3, k, t), total=False)


@pytest.mark.parametrize("name", FLOATS)
@pytest.mark.parametrize("m, k", [(300, 100), (1100, 512), (300, 4096), (600, 3001), (2100, 1000), (257, 12000)])
def test_norm_of_many_rows(T, m, k, name):
    g = rng(k + m)
    t = FLOATS[name]
    check_norm(T, values(g, m, k, t), values(g, m, k, t), (1 + 0.2 * torch.randn(k, generator=g)).to(t))


@pytest.mark.parametrize("name", FLOATS)
@pytest.mark.parametrize("k", [5, 256, 1001, 4096, 20000])
def test_norm_strides_alignment_and_in_place(T, k, name):
    g = rng(k)
    t = FLOATS[name]
    for pad, lead in ((1, 0), (0, 1), (3, 5), (8, 8)):
        x, r, w = values(g, 5, k, t), values(g, 5, k, t), values(g, 1, k, t)[0]
        for in_place in (None, "x", "residual"):
            check_norm(T, x, r, w, pad=pad, lead=lead, in_place=in_place)


@pytest.mark.parametrize("k", [40, 300, 5000, 30001])
def test_norm_of_large_small_and_empty_rows(T, k):
    g = rng(k)
    x = values(g, 6, k, torch.float32)
    x[1] *= 2.0 ** 100        # squares leave the f32 range, and so does their mean
    x[2] *= 2.0 ** -90        # squares vanish beside eps
    x[3] = 0
    x[4] = 0
    x[4, k // 2] = 3.0        # one value alone
    check_norm(T, x, weight=torch.ones(k), eps=1e-20)
    q, scale = torch.empty(6, k, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    T.bnn_rms_norm_clear(x.cuda(), None, 1e-5, q, scale)
    assert float(scale[3]) == 0 and not bool(q[3].any()) and int(q[4, k // 2]) == 127 and int(q[4].abs().sum()) == 127


@pytest.mark.parametrize("name", FLOATS)
def test_rows_that_are_not_numbers(T, name):
    """Rows with an infinity or NaN, anywhere, have scales that are not finite and q = 0; other rows are as without them."""
    t, k = FLOATS[name], 700
    x = values(rng(4), 6, k, t)
    q, scale = torch.empty(6, k, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    q2, scale2 = torch.empty_like(q), torch.empty_like(scale)
    for run in (lambda x, q, s: T.bnn_rms_norm_clear(x, None, 1e-5, q, s), lambda x, q, s: T.bnn_gate_clear(x, None, "identity", q, s)):
        run(x.cuda(), q, scale)
        bad = x.clone()
        bad[0, 0], bad[2, k - 1], bad[4, 333] = math.inf, math.nan, -math.inf
        run(bad.cuda(), q2, scale2)
        for i in range(6):
            if i % 2 == 0:
                assert not math.isfinite(float(scale2[i])) and not bool(q2[i].any())
            else:
                assert torch.equal(q2[i], q[i]) and torch.equal(scale2[i], scale[i])


def act_64(name, v):
    return {"identity": lambda: v, "relu": lambda: v.clamp(min=0), "silu": lambda: v / (1 + torch.exp(-v)),
            "gelu": lambda: 0.5 * v * torch.erfc(-v * math.sqrt(0.5))}[name]()


def act_error(name, v):
    """Relative error of an f32 evaluation in units of u: silu a handful of operations of an ulp or two each; gelu the same, and the
    rounding of erfc's argument z = v / sqrt(2), which erfc(z) ~ exp(-z^2) turns into 2 z^2 = v^2 of them on the negative side."""
    return {"identity": 0 * v, "relu": 0 * v, "silu": 0 * v + 12, "gelu": 24 + 3 * torch.where(v < 0, v * v, 0 * v)}[name]


def check_gate(T, gate, up, act, pad=0, lead=0):
    m, k = gate.shape
    q, scale = strided(torch.zeros(m, k, dtype=torch.int8), pad, lead), torch.empty(m, device="cuda")
    T.bnn_gate_clear(strided(gate, pad, lead), None if up is None else strided(up, 2 * pad, lead), act, q, scale)
    v = gate.double()
    y = act_64(act, v) * (1 if up is None else up.double())
    check_8bit(y, (act_error(act, v) + 1) * U * y.abs() + 2.0 ** -126, q.cpu(), scale.cpu())


@pytest.mark.parametrize("name", FLOATS)
@pytest.mark.parametrize("k", LENGTHS)
def test_gate_lengths(T, k, name):
    g = rng(k)
    t = FLOATS[name]
    for act, up in (("silu", True), ("gelu", True), ("relu", False), ("identity", False), ("silu", False)):
        gate = (3 * torch.randn(4, k, generator=g)).to(t)
        check_gate(T, gate, values(g, 4, k, t) if up else None, act)
    check_gate(T, (3 * torch.randn(1, k, generator=g)).to(t), values(g, 1, k, t), "gelu")


@pytest.mark.parametrize("act", ["identity", "relu", "silu", "gelu"])
@pytest.mark.parametrize("m, k", [(300, 100), (1100, 512), (300, 4096), (600, 3001), (2100, 1000), (257, 12000)])
def test_gate_of_many_rows(T, m, k, act):
    g = rng(k)
    check_gate(T, (2 * torch.randn(m, k, generator=g)).bfloat16(), values(g, m, k, torch.bfloat16), act)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gate_far_from_zero(T, act):
    """Rows of one sign far out, where 1 + erf and 1 / (1 + exp) keep nothing of the value unless they are computed for it."""
    rows = [torch.linspace(a, b, 500) for a, b in ((-12.5, -9), (-9, -4), (-4, -1), (-1, 0), (0, 1), (1, 30), (50, 90), (-80, -20), (-1e-30, 1e-30))]
    gate = torch.stack(rows)
    for i in range(len(rows)):
        if act == "gelu" and float(gate[i].min()) < -13:
            continue            # below the f32 range altogether
        check_gate(T, gate[i:i + 1], None, act)
    low = torch.full((2, 64), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16)    # a mask's value: nothing of it passes
    low[1, 3] = 2
    q, scale = torch.empty(2, 64, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    T.bnn_gate_clear(low.cuda(), None, act, q, scale)
    assert float(scale[0]) == 0 and not bool(q[0].any()) and int(q[1, 3]) == 127 and int(q[1].abs().sum()) == 127


def test_gate_strides_halves_of_one_tensor(T):
    g = rng(1)
    both = (2 * torch.randn(9, 2 * 1234, generator=g)).half()
    d = both.cuda()
    q, scale = torch.empty(9, 1234, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    T.bnn_gate_clear(d[:, :1234], d[:, 1234:], "silu", q, scale)
    q2, scale2 = torch.empty_like(q), torch.empty_like(scale)
    T.bnn_gate_clear(d[:, :1234].contiguous(), d[:, 1234:].contiguous(), "silu", q2, scale2)
    assert torch.equal(q, q2) and torch.equal(scale, scale2)
    for pad, lead in ((1, 0), (0, 1), (3, 5)):
        check_gate(T, both[:, :1001].contiguous(), both[:, 1234:2235].contiguous(), "gelu", pad, lead)


def test_rows_near_the_ends_of_f32(T):
    for s in (2.0 ** -149, 2.0 ** -130, 2.0 ** -101, 2.0 ** -99, 2.0 ** 120):
        v = torch.tensor([[1.0, -64.0, 127.0, 0.0, 30.0]]) * s
        q, scale = torch.empty(1, 5, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
        T.bnn_gate_clear(v.cuda(), None, "identity", q, scale)
        assert q.cpu().tolist() == [[1, -64, 127, 0, 30]] and float(scale) == s


@pytest.mark.parametrize("m, k", [(4_300_000, 3), (1_100_000, 600)])
def test_rows_more_than_a_launch_takes(T, m, k):
    x = (torch.arange(m, device="cuda") % 101 + 1).half()[:, None].expand(m, k).contiguous()
    x[:, 1] = 0
    q, scale = torch.empty(m, k, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    T.bnn_gate_clear(x, None, "identity", q, scale)
    assert bool((q[:, 0] == 127).all()) and bool((q[:, 1] == 0).all()) and bool((q[:, k - 1] == 127).all())
    want = x[:, 0].double() / 127       # 1 / 127 is rounded once, the product with it once
    assert bool(((scale.double() - want).abs() <= 2 * U * (1 + U) * want).all())


# ---- the operators together --------------------------------------------------------------------------------------------

def block(T, s):
    """Norm with the residual, both widening products as one, the gated activation, the narrowing product, the next norm, and a layer
    of signs."""
    T.bnn_rms_norm_clear(s["x"], s["g1"], 1e-5, s["q1"], s["s1"], residual=s["r"], total=s["r"])
    T.bnn_dense_clear(s["q1"], s["w1"], s["wide"], x_scale=s["s1"], w_scale=s["sw1"])
    f = s["wide"].shape[1] // 2
    T.bnn_gate_clear(s["wide"][:, :f], s["wide"][:, f:], "silu", s["q2"], s["s2"])
    T.bnn_dense_clear(s["q2"], s["w2"], s["y"], x_scale=s["s2"], w_scale=s["sw2"], bias=s["b2"])
    T.bnn_rms_norm_clear(s["y"], None, 1e-5, s["q1"], s["s1"], residual=s["r"], total=s["r"])
    T.bnn_dense_clear(s["q1"], s["w3"], s["bits"], bias=s["b3"])


def make_block(m, k, f, p, seed):
    g = rng(seed)
    bf = torch.bfloat16
    s = {"x": torch.randn(m, k, generator=g).to(bf), "r": torch.randn(m, k, generator=g).to(bf), "g1": (1 + 0.1 * torch.randn(k, generator=g)).to(bf),
         "w1": int8(g, 2 * f, k, -127), "sw1": torch.full((2 * f,), 0.0005), "w2": int8(g, k, f, -127), "sw2": torch.full((k,), 0.0007),
         "b2": torch.randn(k, generator=g), "w3": torch.randint(-1, 2, (p, k), generator=g, dtype=torch.int8),
         "b3": torch.randint(-50, 51, (p,), generator=g, dtype=torch.int32)}
    s = {n: v.cuda() for n, v in s.items()}
    for n, shape, t in (("q1", (m, k), torch.int8), ("s1", (m,), torch.float32), ("wide", (m, 2 * f), bf), ("q2", (m, f), torch.int8),
                        ("s2", (m,), torch.float32), ("y", (m, k), bf), ("bits", (m, p), torch.uint8)):
        s[n] = torch.empty(shape, dtype=t, device="cuda")
    return s


@pytest.mark.parametrize("m, k, f, p", [(1, 256, 640, 64), (5, 1001, 333, 20), (70, 512, 1024, 128)])
def test_block_follows_its_formulas(T, m, k, f, p):
    """Each step against its formula on what the step before gave: products and norms compose, strides and types included."""
    s = make_block(m, k, f, p, m)
    before = s["r"].cpu().double() + s["x"].cpu().double()
    block(T, s)
    c = {n: v.cpu() for n, v in s.items()}
    r1 = before.to(torch.float32).to(torch.bfloat16)
    h = r1.double() + c["y"].double()
    # the second residual sum was taken from the stored first one
    assert bool(((c["r"].double() - h).abs() <= (2.0 ** -8 + U) * h.abs()).all())
    y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-5)
    check_8bit(y, 3 * U * y.abs(), c["q1"], c["s1"])
    assert torch.equal(c["bits"].bool(), (c["q1"].double() @ c["w3"].double().t() + c["b3"]) >= 0)
    want = (c["q2"].double() @ c["w2"].double().t()) * c["s2"].double()[:, None] * c["sw2"].double() + c["b2"].double()
    assert bool(((c["y"].double() - want).abs() <= 2.0 ** -8 * want.abs() + 4 * U * (want - c["b2"]).abs() + 1e-30).all())
    v = c["wide"].double()
    gated = act_64("silu", v[:, :f]) * v[:, f:]
    check_8bit(gated, 13 * U * gated.abs() + 2.0 ** -126, c["q2"], c["s2"])


def test_block_captured_replayed_and_on_another_stream(T):
    """A captured block replayed on new inputs, with eager calls and a second captured block between, on a stream of its own: the bytes
    of the eager calls each time."""
    a, b = make_block(9, 384, 512, 40, 1), make_block(3, 256, 300, 17, 2)
    graphs = []
    for s in (a, b):
        block(T, s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            block(T, s)
        graphs.append(graph)
    side = torch.cuda.Stream()
    for turn in range(4):
        for s, graph, shape in ((a, graphs[0], (9, 384, 512, 40)), (b, graphs[1], (3, 256, 300, 17))):
            new = make_block(*shape, 50 + turn)
            for n in ("x", "r", "w1"):
                s[n].copy_(new[n])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for s, shape in ((a, (9, 384, 512, 40)), (b, (3, 256, 300, 17))):
            new = make_block(*shape, 50 + turn)
            want = {n: new[n] if n in ("x", "r", "w1") else s[n].clone() for n in s}
            with torch.cuda.stream(side):
                block(T, want)
            torch.cuda.synchronize()
            for n in ("r", "q1", "s1", "wide", "q2", "s2", "y", "bits"):
                assert torch.equal(s[n], want[n]), (turn, n)


def test_clear_layer_of_signs_is_the_encrypted_layer(T):
    """Real features to bits by an 8-bit layer in the clear, the bits encrypted, two binary layers on ciphertexts: the answers decrypt to
    what the same layers give in the clear."""
    import numpy as np
    import workloads
    g = rng(12)
    d, p1, p2 = 24, 8, 3
    features = torch.randn(1, 50, generator=g)
    q, s = torch.empty(1, 50, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    T.bnn_rms_norm_clear(features.cuda(), None, 1e-5, q, s)
    bits = torch.empty(1, d, dtype=torch.uint8, device="cuda")
    T.bnn_dense_clear(q, int8(g, d, 50).cuda(), bits)
    W1, W2 = (torch.randint(-1, 2, shape, generator=g, dtype=torch.int8) for shape in ((p1, d), (p2, p1)))
    thresholds = [torch.randint(3, 6, (w.shape[0],), generator=g, dtype=torch.int32) for w in (W1, W2)]
    # in the clear: signs, with bias = (non-zero weights) - 2 T
    h = (2 * bits.to(torch.int8) - 1)
    clear = []
    for w, t in zip((W1, W2), thresholds):
        out = torch.empty(1, w.shape[0], dtype=torch.int8, device="cuda")
        T.bnn_dense_clear(h, w.cuda(), out, bias=((w != 0).sum(dim=1).to(torch.int32) - 2 * t).cuda())
        clear.append(out)
        h = out
    sk, ck = T.tfhe_keygen(T.default_params(), workloads.KEY_SEED)
    c = T.to_device(T.tfhe_encrypt(sk, 8, bits.cpu().numpy()))
    for w, t, want in zip((W1, W2), thresholds, clear):
        out = torch.empty(w.shape[0], 501, dtype=torch.int32, device="cuda")
        T.bnn_dense_encrypted(ck, c, w.shape[1], w.numpy(), t.numpy(), w.shape[0], out)
        torch.cuda.synchronize()
        assert np.array_equal(T.tfhe_decrypt(sk, T.to_host(out)), (want.cpu().numpy().ravel() + 1) // 2)
        c = out


# ---- refusals of the binding ---------------------------------------------------------------------------------------------

def test_binding_refuses_what_does_not_fit(T):
    z = lambda *s, t=torch.int8: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
    x, w, out = z(2, 8), z(4, 8), z(2, 4, t=torch.float32)
    for bad in (dict(x=z(2, 9)), dict(x=z(3, 8)), dict(x=z(2, 8, t=torch.uint8)), dict(x=z(8)), dict(w=z(4, 9)), dict(w=z(5, 8)), dict(x=z(8, 2).t()),
                dict(x=z(2, 8).cpu()), dict(x=z(1, 8).expand(2, 8)), dict(x_scale=z(3, t=torch.float32)), dict(x_scale=z(2, t=torch.float64)),
                dict(w_scale=z(2, t=torch.float32)), dict(bias=z(4, t=torch.int32)), dict(w_scale=z(8, t=torch.float32)[::2]),
                dict(out=z(2, 4, t=torch.int32), bias=z(4, t=torch.float32)), dict(out=z(4, 2, t=torch.float32).t()), dict(out=z(2, 4, 1, t=torch.float32))):
        with pytest.raises(ValueError):
            T.bnn_dense_clear(**dict(dict(x=x, w=w, out=out), **bad))
    for dtype in (torch.float64, torch.int64, torch.bool):
        with pytest.raises(T.TfheError):
            T.bnn_dense_clear(x, w, z(2, 4, t=dtype))
    with pytest.raises(T.TfheError):
        T.bnn_dense_clear(x, w, z(2, 4, t=torch.int32), x_scale=z(2, t=torch.float32))
    f, q, s = z(2, 8, t=torch.bfloat16), z(2, 8), z(2, t=torch.float32)
    for bad in (dict(weight=z(8, t=torch.float32)), dict(weight=z(7, t=torch.bfloat16)), dict(residual=z(2, 8, t=torch.half)), dict(total=z(2, 7, t=torch.bfloat16)),
                dict(q=z(2, 8, t=torch.uint8)), dict(scale=z(2, t=torch.float64))):
        with pytest.raises(ValueError):
            T.bnn_rms_norm_clear(**dict(dict(x=f, weight=None, eps=1e-5, q=q, scale=s), **bad))
    with pytest.raises(T.TfheError):
        T.bnn_rms_norm_clear(q, None, 1e-5, q, s)
    with pytest.raises(ValueError):
        T.bnn_gate_clear(f, None, "tanh", q, s)
    with pytest.raises(ValueError):
        T.bnn_gate_clear(f, z(2, 8, t=torch.float32), "silu", q, s)
