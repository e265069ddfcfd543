"""GPU tests of the 8-bit product where a workgroup takes more than one tile.

A launch has 2^20 workgroups at most.  Which tiles a size gets goes by what a launch of each takes; the sizes here are such that each form that can have more tiles
than that has them: 64 x 64 (few channels), 256 x 128 (few channels and short rows, or rows at any address), 256 x 256.  The others never do: for so many tiles
larger ones always take less.  Operands repeat with prime periods, so the expected outputs are a small product repeated, and a tile that kept anything
of the one before it shows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    import paper_1806_03461_amd
    return paper_1806_03461_amd


def repeated(base, rows):
    p = base.shape[0]
    out = torch.empty((rows,) + base.shape[1:], dtype=base.dtype, device="cuda")
    whole = rows // p * p
    out[:whole].view(-1, *base.shape).copy_(base)
    out[whole:] = base[:rows - whole]
    return out


@pytest.mark.parametrize("m, n, k, out", [
    (67_200_001, 61, 132, "f32"),           # 64 x 64, straight to LDS
    (67_200_001, 61, 259, "i32"),           # 64 x 64, through registers
    (268_600_000, 127, 4, "sign"),          # 256 x 128, straight
    (262_300, 131_100, 451, "f16"),         # 256 x 128, through registers
    (262_300, 262_200, 516, "bits")])       # 256 x 256, straight
def test_product_of_more_tiles_than_workgroups(T, m, n, k, out):
    g = torch.Generator(device="cuda").manual_seed(k)
    pm, pn = min(1009, m), min(997, n)
    xs, ws = (torch.randint(-128, 128, (r, k), generator=g, device="cuda", dtype=torch.int8) for r in (pm, pn))
    acc = xs.double() @ ws.double().t()
    scales, bias = {}, None
    if out in ("f32", "f16"):
        # powers of two and whole numbers: in units of the product of its scales, 2^-15 at least, an output is acc + b 2^15 at most, at most
        # 2^14 * 451 + 2^18 < 2^24, so every step is exact in f32; f16 rounds once
        sx, sw = (torch.exp2(torch.randint(-3, 1, (r,), generator=g, device="cuda").float()) for r in (pm, pn))
        sw = sw * 2.0 ** -9
        b = torch.randint(-8, 9, (pn,), generator=g, device="cuda").float()
        scales, bias = {"x_scale": repeated(sx, m), "w_scale": repeated(sw, n)}, repeated(b, n)
        want = (acc * sx.double()[:, None] * sw.double() + b.double()).to({"f32": torch.float32, "f16": torch.float16}[out])
    else:
        b = torch.randint(-3000, 3000, (pn,), generator=g, device="cuda", dtype=torch.int32)
        bias, total = repeated(b, n), acc + b.double()
        want = total.to(torch.int32) if out == "i32" else torch.where(total >= 0, 1, -1).to(torch.int8) if out == "sign" else (total >= 0).to(torch.uint8)
    got = torch.empty(m, n, dtype=want.dtype, device="cuda")
    T.bnn_dense_clear(repeated(xs, m), repeated(ws, n), got, bias=bias, **scales)
    want = repeated(want.t().contiguous(), n).t().contiguous()      # [pm][n]
    each = max(1, (1 << 30) // (pm * n)) * pm
    for i in range(0, m, each):
        part = got[i:i + each]
        whole = part.shape[0] // pm * pm
        assert bool((part[:whole].view(-1, pm, n) == want).all()) and torch.equal(part[whole:], want[:part.shape[0] - whole]), i
    del got, part
    torch.cuda.empty_cache()
