"""The work memory of a table's gradient, checked without a GPU: none is asked for or
allocated where no kernel reads it."""
import os

import pytest

from paper_2407_15264_amd import lsmgnn


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lsmgnn.LIB_PATH):
        from paper_2407_15264_amd import build
        build.build_hip()
    return lsmgnn.lib()


@pytest.mark.parametrize("n,num_rows,dim,some", [
    (1, 256, 8, False), (12288, 1 << 24, 65536, False), (9001, 16384, 128, False), (0, 1000, 8, False),
    (12289, 1 << 20, 8, True), (5, 255, 8, True), (5, (1 << 24) + 1, 8, True)])
def test_whole_gradient(L, n, num_rows, dim, some):
    either = lsmgnn.embed_grad_work_bytes(n, num_rows, dim)
    assert lsmgnn.table_grad_work_bytes(n, num_rows, dim) == (either if some else 0)
    assert bool(either) == bool(n)


def test_it_is_what_the_call_takes(L):
    a = 1 << 20  # never read: these calls are refused
    need = lsmgnn.table_grad_work_bytes(20000, 1000, 8)
    args = dict(dy=a, dim=8, ld=8, type=0, ids=a, n=20000, num_rows=1000, pad=-1, scale=1.0, grad=a, grad_ld=8,
                grad_type=0, work=a, work_bytes=need, status=None, stream=None)
    for change in (dict(work=None), dict(work=a + 16), dict(work_bytes=need - 1)):
        assert L.lsmgnn_embed_grad(*dict(args, **change).values()) == lsmgnn.E_INVAL


@pytest.mark.gpu
def test_whole_gradient_of_few_places_takes_no_memory():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dy = torch.ones((12288, 1024), device="cuda")
    ids = torch.arange(12288, device="cuda") % 3
    grad = torch.empty((300, 1024), device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    lsmgnn.embed_grad(dy, ids, 300, grad=grad)
    assert torch.cuda.max_memory_allocated() == before
    assert bool((grad[:3] == 4096).all()) and not grad[3:].any()
