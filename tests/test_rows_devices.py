"""The operators on trained rows with tensors of a device that is not the current one,
checked without a GPU: the binding calls the library with the tensors' device current,
since a default stream's handle names the current device's, and refuses memory and
streams of another."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2407_15264_amd import lsmgnn  # noqa: E402

CALLS = ["embed_rows", "embed_grad", "embed_grad_rows", "route_plan", "route_rows", "route_combine",
         "route_combine_grad", "pack8", "unpack8", "act8", "act8_grad", "weight_grad8"]


class OnSecond(torch.Tensor):
    """A host tensor that says it is on the second device."""
    is_cuda = True
    device = torch.device("cuda", 1)


class OnFirst(torch.Tensor):
    is_cuda = True
    device = torch.device("cuda", 0)


def second(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnSecond)


@pytest.fixture
def calls(monkeypatch):
    """What the library is called with: (name, the current device, the stream)."""
    made, now = [], [0]

    class Guard:
        def __init__(self, device):
            self.device = torch.device(device).index

        def __enter__(self):
            self.before, now[0] = now[0], self.device

        def __exit__(self, *_):
            now[0] = self.before

    fake = types.SimpleNamespace(lsmgnn_route_max_rows=lambda n, k, num, align: n * k,
                                 lsmgnn_route_work_bytes=lambda *a: 256, lsmgnn_embed_grad_work_bytes=lambda *a: 256,
                                 lsmgnn_table_grad_work_bytes=lambda *a: 256,
                                 lsmgnn_weight_grad8_work_bytes=lambda *a: 256)
    for name in CALLS:
        setattr(fake, "lsmgnn_" + name,
                lambda *a, name=name: made.append((name, now[0], a[-1])) or lsmgnn.OK)
    monkeypatch.setattr(lsmgnn, "lib", lambda: fake)
    monkeypatch.setattr(lsmgnn, "_empty", lambda shape, dtype, device, stream: torch.zeros(
        shape, dtype=dtype).as_subclass(OnSecond))
    monkeypatch.setattr(lsmgnn, "_raw_stream", lambda index: 1000 * index)
    monkeypatch.setattr(lsmgnn, "_raw_device", lambda: now[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    return made


def run_all(**kw):
    i64 = torch.int64
    x, ids = second(4, 8), second(4, dtype=i64)
    lsmgnn.embed_rows(x, ids, **kw)
    lsmgnn.embed_grad(x, ids, 10, **kw)
    lsmgnn.embed_grad_rows_async(x, ids, 10, second(4, dtype=i64), second(4, 8), 0, **kw)
    plan = lsmgnn.route_plan(second(4, 2, dtype=i64), 3, **kw)
    rows, w = lsmgnn.route_rows(x, plan, **kw), second(4, 2)
    lsmgnn.route_combine(rows, plan, w, **kw)
    lsmgnn.route_combine_grad(x, rows, plan, w, **kw)
    kept = lsmgnn.pack8(x, **kw)
    lsmgnn.unpack8(kept, **kw)
    y, kept = lsmgnn.act8(x, "gelu", **kw)
    lsmgnn.act8_grad(y, kept, "gelu", **kw)
    lsmgnn.weight_grad8(kept, y, **kw)


def test_the_tensors_device_is_current(calls):
    run_all()
    assert calls == [(name, 1, 1000) for name in CALLS]


def test_with_a_stream_of_it(calls):
    run_all(stream=types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=77))
    assert calls == [(name, 1, 77) for name in CALLS]


def test_a_stream_of_another_device_is_refused(calls):
    stream = types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=77)
    with pytest.raises(ValueError, match="stream"):
        lsmgnn.embed_rows(second(4, 8), second(4, dtype=torch.int64), stream=stream)
    assert not calls


def test_work_of_another_device_is_refused(calls):
    work = torch.zeros(1024, dtype=torch.uint8).as_subclass(OnFirst)
    x, ids = second(4, 8), second(4, dtype=torch.int64)
    for call in (lambda: lsmgnn.embed_grad(x, ids, 10, work=work),
                 lambda: lsmgnn.route_plan(ids.view(2, 2), 4, work=work),
                 lambda: lsmgnn.weight_grad8(lsmgnn.Packed8(4, 8, OnSecond.device), x, work=work)):
        with pytest.raises(ValueError, match="work"):
            call()
    assert not calls
