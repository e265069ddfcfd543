"""GPU tests of layers in the clear: products of many steps of k, what a product promises of a row's bytes, and what lies around the rows that the
row operators write."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    import paper_1806_03461_amd
    return paper_1806_03461_amd


@pytest.mark.parametrize("m, n", [(4625, 1665), (300, 5000), (3285, 587), (2049, 1000), (97, 161), (898, 4435), (4663, 2562)])
@pytest.mark.parametrize("more", [0, 1])
def test_product_of_many_steps(T, m, n, more):
    """Ten to twenty-five steps of 128 bytes, whole and not, for 64 x 128 tiles (the first two), 128 x 128 (the next two), 32 x 64, 256 x 128 and
    256 x 256: their loops without conditions go round more than once.  At rows of multiples of 4 bytes and at any."""
    g = torch.Generator(device="cuda").manual_seed(m + more)
    for k in (1280, 1284, 1408, 1536, 1600, 1664, 1792, 1924, 2048, 2304, 2500, 2560, 2688, 3200):
        k += more
        x, w = (torch.randint(-128, 128, (r, k), generator=g, device="cuda", dtype=torch.int8) for r in (m, n))
        wide = torch.full((m + 1, n + 3), -7, dtype=torch.int32, device="cuda")
        T.bnn_dense_clear(x, w, wide[:m, :n])
        assert torch.equal(wide[:m, :n].double(), x.double() @ w.double().t()), k
        assert bool((wide[m] == -7).all()) and bool((wide[:, n:] == -7).all()), k


@pytest.mark.parametrize("k", [100, 1024, 1001])
def test_rows_of_a_product_do_not_depend_on_the_others(T, k):
    """The same rows among 1 to 2,000 tokens and 40 to 700 channels, by every kernel and form that takes such sizes: the same bytes."""
    g = torch.Generator(device="cuda").manual_seed(k)
    x, w = (torch.randint(-128, 128, (r, k), generator=g, device="cuda", dtype=torch.int8) for r in (2000, 700))
    sx, sw, b = torch.randn(2000, generator=g, device="cuda"), torch.randn(700, generator=g, device="cuda"), torch.randn(700, generator=g, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        full = torch.empty(2000, 700, dtype=dtype, device="cuda")
        T.bnn_dense_clear(x, w, full, x_scale=sx, w_scale=sw, bias=b)
        for m, n in ((1, 700), (3, 40), (16, 700), (31, 300), (33, 700), (100, 64), (300, 129), (700, 700), (1500, 500)):
            i, j = (2000 - m) // 2, (700 - n) // 2
            part = torch.empty(m, n, dtype=dtype, device="cuda")
            T.bnn_dense_clear(x[i:i + m], w[j:j + n], part, x_scale=sx[i:i + m].clone(), w_scale=sw[j:j + n].clone(), bias=b[j:j + n].clone())
            assert torch.equal(part, full[i:i + m, j:j + n]), (m, n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m, k", [(5, 1), (9, 90), (6, 511), (7, 1001), (1030, 4097), (5, 12000), (3, 16390), (3, 32765)])
def test_row_operators_write_rows_and_nothing_else(T, m, k, dtype):
    """q, total and scale among values that stay: between the rows, in front of the first and behind the last."""
    g = torch.Generator(device="cuda").manual_seed(k)
    x, r = (torch.randn(m, k, generator=g, device="cuda").to(dtype) for _ in range(2))
    for pad, lead in ((1, 0), (5, 3), (8, 8)):
        def among(t):
            flat = torch.full((lead + (m + 1) * (k + pad),), 77, dtype=t, device="cuda")
            return flat, torch.as_strided(flat, (m, k), (k + pad, 1), lead)
        for norm in (True, False):
            (fq, q), (ft, total) = among(torch.int8), among(dtype)
            fs = torch.full((m + 2,), 77.0, device="cuda")
            if norm:
                T.bnn_rms_norm_clear(x, None, 1e-5, q, fs[1:m + 1], residual=r, total=total)
                assert torch.equal(total, (x.float() + r.float()).to(dtype))
                total.fill_(77)
            else:
                T.bnn_gate_clear(x, r, "gelu", q, fs[1:m + 1])
            assert int(q.max()) <= 127 and bool((q.abs().amax(dim=1) == 127).all())
            q.fill_(77)
            assert bool((fq == 77).all()) and bool((ft == 77).all())
            assert fs[0] == 77 and fs[m + 1] == 77 and not bool((fs[1:m + 1] == 77).any())
