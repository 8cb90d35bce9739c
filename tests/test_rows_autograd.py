"""The operators on trained rows and torch's differentiation: they record nothing, so a
tensor that requires a gradient is refused where torch would record, and accepted under
no_grad and in an autograd.Function's own passes."""
import pytest

from tests.test_rows_devices import calls, second  # noqa: F401

torch = pytest.importorskip("torch")

from paper_2407_15264_amd import lsmgnn  # noqa: E402


def requests():
    """name of the argument -> a call with one that requires a gradient"""
    i64 = torch.int64
    leaf = lambda *s: second(*s).requires_grad_()  # noqa: E731
    ids = second(4, dtype=i64)
    plan = lsmgnn.RoutePlan(4, 2, 3, 1, 8, second(1).device, None)
    kept = lsmgnn.Packed8(4, 8, second(1).device)
    return [("table", lambda: lsmgnn.embed_rows(leaf(4, 8), ids)),
            ("dy", lambda: lsmgnn.embed_grad(leaf(4, 8), ids, 10)),
            ("grad", lambda: lsmgnn.embed_grad(second(4, 8), ids, 10, grad=leaf(10, 8))),
            ("x", lambda: lsmgnn.route_rows(leaf(4, 8), plan)),
            ("z", lambda: lsmgnn.route_combine(leaf(8, 8), plan)),
            ("weights", lambda: lsmgnn.route_combine(second(8, 8), plan, leaf(4, 2))),
            ("x", lambda: lsmgnn.pack8(leaf(4, 8))),
            ("x", lambda: lsmgnn.act8(leaf(4, 8), "silu")),
            ("dy", lambda: lsmgnn.act8_grad(leaf(4, 8), kept, "silu")),
            ("dy", lambda: lsmgnn.weight_grad8(kept, leaf(4, 8)))]


def test_refused_where_torch_records(calls):  # noqa: F811
    for name, call in requests():
        with pytest.raises(RuntimeError, match=f"^{name} requires a gradient"):
            call()
    assert not calls


def test_accepted_where_it_does_not(calls):  # noqa: F811
    with torch.no_grad():
        for _, call in requests():
            call()
    assert len(calls) == len(requests())


@pytest.mark.gpu
def test_in_an_autograd_function():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")

    class Rows(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, ids):
            ctx.save_for_backward(ids)
            ctx.num_rows = table.shape[0]
            return lsmgnn.embed_rows(table, ids, scale=2.0)

        @staticmethod
        def backward(ctx, dy):
            return lsmgnn.embed_grad(dy.contiguous(), *ctx.saved_tensors, ctx.num_rows, scale=2.0), None

    table = torch.randn(9, 5, device="cuda", requires_grad=True)
    ids = torch.tensor([3, 1, 3, 8], device="cuda")
    w = torch.randn(4, 5, device="cuda")
    (Rows.apply(table, ids) * w).sum().backward()
    want = torch.zeros(9, 5, device="cuda").index_add_(0, ids, 2 * w)
    assert torch.allclose(table.grad, want, rtol=1e-6, atol=1e-6)
