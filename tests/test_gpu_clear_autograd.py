"""GPU tests: layers in the clear have no gradients.  With gradients recorded, an operand that asks for one is refused rather than
cut off from its graph, and what a call writes is marked as written, so that a backward pass that saved it says so."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def T():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    import paper_1806_03461_amd
    return paper_1806_03461_amd


def operands():
    g = torch.Generator(device="cuda").manual_seed(5)
    f = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    i = lambda *s: torch.randint(-128, 128, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    return {"bnn_dense_clear": dict(x=i(6, 40), w=i(9, 40), out=f(6, 9), x_scale=f(6), w_scale=f(9), bias=f(9)),
            "bnn_rms_norm_clear": dict(x=f(6, 40), weight=f(40), eps=1e-5, q=i(6, 40), scale=f(6), residual=f(6, 40), total=f(6, 40)),
            "bnn_gate_clear": dict(gate=f(6, 40), up=f(6, 40), act="silu", q=i(6, 40), scale=f(6))}


WRITTEN = {"bnn_dense_clear": ("out",), "bnn_rms_norm_clear": ("q", "scale", "total"), "bnn_gate_clear": ("q", "scale")}
CASES = [(name, op) for name, ops in (("bnn_dense_clear", ("out", "x_scale", "w_scale", "bias")), ("bnn_rms_norm_clear", ("x", "weight", "scale", "residual", "total")),
                                      ("bnn_gate_clear", ("gate", "up", "scale"))) for op in ops]


@pytest.mark.parametrize("name, operand", CASES)
def test_operands_that_ask_for_gradients_are_refused(T, name, operand):
    a = operands()[name]
    a[operand].requires_grad_(True)
    before = {n: a[n].detach().clone() for n in WRITTEN[name]}
    with pytest.raises(ValueError, match=operand + ".*gradient"):
        getattr(T, name)(**a)
    torch.cuda.synchronize()
    assert all(torch.equal(a[n], before[n]) for n in before)
    with torch.no_grad():           # asked for without gradients, the same call runs
        getattr(T, name)(**a)
    b = dict(a, **{operand: a[operand].detach().clone()}, **{n: a[n].detach().clone() for n in WRITTEN[name] if n != operand})
    getattr(T, name)(**b)
    for n in WRITTEN[name]:
        assert torch.equal(a[n], b[n]), n


@pytest.mark.parametrize("name", WRITTEN)
def test_what_a_call_writes_is_marked_as_written(T, name):
    a = operands()[name]
    call = getattr(T, name)
    before = {n: t._version for n, t in a.items() if isinstance(t, torch.Tensor)}
    call(**a)
    for n, v in before.items():
        assert (a[n]._version > v) == (n in WRITTEN[name]), n
    with torch.inference_mode():
        call(**{n: t.clone() if isinstance(t, torch.Tensor) else t for n, t in a.items()})


def test_a_backward_pass_that_saved_the_residual_says_so(T):
    a = operands()["bnn_rms_norm_clear"]
    p = torch.ones(40, device="cuda", requires_grad=True)
    y = (a["residual"] * p).sum()               # saves the residual for p's gradient
    T.bnn_rms_norm_clear(a["x"], a["weight"], 1e-5, a["q"], a["scale"], residual=a["residual"], total=a["residual"])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_marks_in_a_captured_block(T):
    """Capturing marks the outputs once more and enqueues nothing for it; replays give the eager bytes."""
    a = operands()["bnn_gate_clear"]
    T.bnn_gate_clear(**a)
    torch.cuda.synchronize()
    want = {n: a[n].clone() for n in ("q", "scale")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.bnn_gate_clear(**a)
    for _ in range(3):
        a["q"].zero_()
        a["scale"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], want[n]) for n in want)
