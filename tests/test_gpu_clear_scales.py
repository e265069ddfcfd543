"""GPU tests: a row's scale is max|y| / 127 in f32, off by half a step at most, and q is y / scale as f32 divides, to the nearest whole number, ties to
even.  Rows whose y is in hand as f32 (identity and relu without a second factor, a norm without weight and residual, where q needs no rms)
therefore follow these two formulas bit for bit; rows of few bits hold values at half the largest, whose quotient is at a tie."""
import pytest
import torch

pytestmark = pytest.mark.gpu

FLOATS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def T():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    import paper_1806_03461_amd
    return paper_1806_03461_amd


def by_formula(y):
    """f32 on the CPU, whose divisions are rounded to the nearest."""
    scale = y.abs().amax(dim=1) / 127
    q = torch.round(torch.where(scale[:, None] > 0, y / scale[:, None], torch.zeros_like(y)))
    return q.to(torch.int8), scale


def rows(m, k, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, k, generator=g) * torch.exp(2 * torch.randn(m, 1, generator=g))
    x = x.to(dtype)
    if k > 2:       # half of each row's largest, of both signs
        top = x.float().abs().amax(dim=1)
        x[:, 0] = (top / 2).to(dtype)
        x[:, k // 2] = (-top / 2).to(dtype)
    return x


@pytest.mark.parametrize("name", FLOATS)
@pytest.mark.parametrize("m, k", [(4000, 1), (3001, 90), (2000, 512), (900, 1001), (1100, 4096), (700, 8192), (600, 12000), (300, 20000), (64, 32768), (40, 65536)])
def test_rows_to_8_bits_by_the_formula(T, m, k, name):
    x = rows(m, k, FLOATS[name], m + k)
    d = x.cuda()
    q, scale = torch.empty(m, k, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    for act, y in (("identity", x.float()), ("relu", x.float().clamp(min=0))):
        T.bnn_gate_clear(d, None, act, q, scale)
        want_q, want = by_formula(y)
        assert torch.equal(scale.cpu(), want), act
        assert torch.equal(q.cpu(), want_q), (act, int((q.cpu() != want_q).sum()))
    if k <= 32768:
        T.bnn_rms_norm_clear(d, None, 1e-5, q, scale)
        want_q, _ = by_formula(x.float())
        assert torch.equal(q.cpu(), want_q), int((q.cpu() != want_q).sum())


def test_every_leading_digit_of_a_largest_value(T):
    """All 2^16 values of bf16 and f16 that are finite numbers, each as a row's largest beside its half and its quarter: those whose scale is a
    normal f32."""
    for dtype in (torch.bfloat16, torch.float16):
        top = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(dtype)
        top = top[torch.isfinite(top.float()) & (top.float().abs() >= 2.0 ** -118)]
        x = torch.stack([top, (top.float() / 2).to(dtype), (-top.float() / 4).to(dtype), torch.zeros_like(top)], dim=1).contiguous()
        q, scale = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(x.shape[0], device="cuda")
        T.bnn_gate_clear(x.cuda(), None, "identity", q, scale)
        want_q, want = by_formula(x.float())
        assert torch.equal(scale.cpu(), want) and torch.equal(q.cpu(), want_q), (int((scale.cpu() != want).sum()), int((q.cpu() != want_q).sum()))


def test_rows_at_the_bottom_of_f32(T):
    """Largest values from 2^-149 to 2^-90: q goes by max / 127 itself, the scale is that number to the nearest f32, of few digits or none down there."""
    g = torch.Generator().manual_seed(3)
    top = torch.exp2(torch.linspace(-149, -90, 4000, dtype=torch.float64))
    x = (top[:, None] * (2 * torch.rand(4000, 300, generator=g, dtype=torch.float64) - 1)).float()
    x[:, 7] = top.float()
    q, scale = torch.empty(4000, 300, dtype=torch.int8, device="cuda"), torch.empty(4000, device="cuda")
    T.bnn_gate_clear(x.cuda(), None, "identity", q, scale)
    want = x[:, 7].double() / 127
    assert torch.equal(scale.cpu(), want.float())
    real = x.double() / want[:, None]
    # the step is one rounding of max / 127 and the quotient by it another, 127 * 2^-23 at most
    assert bool(((q.cpu().double() - real).abs() <= 0.5 + 127 * 2.0 ** -23).all())
    assert bool((q.cpu()[:, 7] == 127).all())
