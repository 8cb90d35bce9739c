"""The operators on trained rows in layouts that the other tests leave out: elements
past 2^32 of a matrix, the caller's own outputs with gaps between their rows, status
words and row counts of captured calls, every type through many experts."""
import numpy as np
import pytest

from tests import rows_reference as ref
from tests.test_gpu_embed import TYPES, ids_of, rows
from tests.test_gpu_packed import check_weight, spread

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2407_15264_amd import lsmgnn  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lsmgnn.lib()


def room_for(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GiB of device memory")


# ----------------------------------------------------------- elements past 2^32
FAR = (1 << 31) + 64  # elements between rows: the third row begins past 2^32


def far_rows(n, dim, dtype):
    """n rows FAR apart, in memory that is not cleared."""
    return torch.empty((n - 1) * FAR + dim, dtype=dtype, device="cuda").as_strided((n, dim), (FAR, 1))


def put(view, rng):
    view.copy_(torch.as_tensor(rng.standard_normal(tuple(view.shape)), dtype=torch.float32).cuda())
    return view


def test_far_rows_of_a_gradient():
    room_for(40)
    rng = np.random.default_rng(1)
    dy = put(far_rows(4, 40, torch.bfloat16), rng)
    ids = np.array([2, 0, 2, 299], np.int64)
    unique, sums, bound = ref.row_sums(ref.f64(dy), ids, 300, 1.0, None)
    got_ids, got = lsmgnn.embed_grad_rows(dy, torch.as_tensor(ids).cuda(), 300)
    assert np.array_equal(got_ids.cpu().numpy(), unique)
    ref.assert_within(got, sums, bound, torch.bfloat16)
    # rows of the gradient: 300 of them, 2^24 apart; one launch, and the sort's
    for n in (4, 13000):
        grad = torch.empty(299 * (1 << 24) + 40, dtype=torch.bfloat16, device="cuda").as_strided((300, 40), (1 << 24, 1))
        near = rows(rng, n, 40, torch.bfloat16)
        many = ids_of(rng, n, 300)
        lsmgnn.embed_grad(near, torch.as_tensor(many).cuda(), 300, grad=grad)
        unique, sums, bound = ref.row_sums(ref.f64(near), many, 300, 1.0, None)
        want, allow = np.zeros((300, 40)), np.zeros((300, 40))
        want[unique], allow[unique] = sums, bound
        ref.assert_within(grad, want, allow, torch.bfloat16)
        del grad
    out = far_rows(4, 40, torch.bfloat16)
    table = rows(rng, 300, 40, torch.bfloat16)
    lsmgnn.embed_rows(table, torch.as_tensor(ids).cuda(), out=out)
    assert torch.equal(out, table[torch.as_tensor(ids).cuda()])


def test_far_rows_by_expert():
    room_for(80)
    rng = np.random.default_rng(2)
    e = np.array([[1, 0], [0, -1], [1, 1], [0, 1]], np.int64)
    w = rng.random((4, 2)).astype(np.float32)
    p = lsmgnn.route_plan(torch.as_tensor(e).cuda(), 2)
    _, slot, source = ref.plan(e, 2, 1)
    x, d_w = put(far_rows(4, 24, torch.float16), rng), torch.as_tensor(w).cuda()
    z = lsmgnn.route_rows(x, p, out=far_rows(8, 24, torch.float16))
    assert np.array_equal(ref.f64(z), ref.sorted_rows(ref.f64(x), source, 2))
    y, bound = ref.combine(ref.f64(z), slot, w.astype(np.float64))
    ref.assert_within(lsmgnn.route_combine(z, p, d_w, out=far_rows(4, 24, torch.float16)), y, bound, torch.float16)
    dz, bz, dw, bw = ref.combine_grad(ref.f64(x), ref.f64(z), slot, source, w.astype(np.float64))
    got_dz, got_dw = lsmgnn.route_combine_grad(x, z, p, d_w, dz=far_rows(8, 24, torch.float16))
    ref.assert_within(got_dz, dz, bz, torch.float16)
    ref.assert_within(got_dw, dw, bw, torch.float32)


def test_kept_rows_past_two_to_the_32():
    """70000 rows of 65536 whole numbers, which are kept exactly."""
    room_for(60)
    n, dim = 70_000, 65_536
    x = torch.empty((n, dim), dtype=torch.bfloat16, device="cuda")
    for a in range(0, n, 10_000):
        x[a:a + 10_000] = torch.randint(-64, 65, (10_000, dim), dtype=torch.int8, device="cuda")
    p = lsmgnn.pack8(x)
    out = lsmgnn.unpack8(p, out=torch.full_like(x, 3.0))
    for a in range(0, n, 10_000):
        assert torch.equal(out[a:a + 10_000], x[a:a + 10_000])
    y, p = lsmgnn.act8(x, "silu", gated=True, out=out.view(-1)[:n * dim // 2].view(n, dim // 2))
    part = slice(n - 50, n)
    want, kept = lsmgnn.act8(x[part], "silu", gated=True)
    assert torch.equal(y[part], want)
    dx = lsmgnn.act8_grad(y, p, "silu", gated=True)
    assert torch.equal(dx[part], lsmgnn.act8_grad(want, kept, "silu", gated=True))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_gradient_of_rows_past_two_to_the_32(dtype):
    """Small whole numbers, whose sums 32 bits hold exactly."""
    room_for(60)
    n, din, dout = 4_400_000, 1024, 40
    x = torch.empty((n, din), dtype=torch.bfloat16, device="cuda")
    dy = torch.randint(-1, 2, (n, dout), dtype=torch.int8, device="cuda").to(dtype)
    want = torch.zeros((2, din, dout), device="cuda")
    cut = 4_300_001
    for a in range(0, n, 100_000):
        x[a:a + 100_000] = torch.randint(-1, 2, (100_000, din), dtype=torch.int8, device="cuda")
        for e, (lo, hi) in enumerate(((a, min(a + 100_000, cut)), (max(a, cut), a + 100_000))):
            if hi > lo:
                want[e] += torch.mm(x[lo:hi].float().t().contiguous(), dy[lo:hi].float())
    p = lsmgnn.pack8(x)
    got = lsmgnn.weight_grad8(p, dy, torch.tensor([0, cut, n], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, want)


# ------------------------------------------------------------ the caller's outputs
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", [False, True])
def test_activation_into_outputs_with_gaps(dtype, gated):
    rng, n, dim, parts = np.random.default_rng(5), 60, 75, 2 if gated else 1
    x, dy = spread(rng, n, dim * parts, dtype), rows(rng, n, dim, dtype)
    want, kept = lsmgnn.act8(x, "gelu", gated)
    want_dx = lsmgnn.act8_grad(dy, kept, "gelu", gated)

    def gaps(width):
        flat = torch.full((n * (width + 7) + 3,), 9.0, dtype=dtype, device="cuda")
        return flat, flat[3:].view(n, width + 7)[:, :width]

    flat, out = gaps(dim)
    packed = lsmgnn.Packed8(n * parts, dim, x.device)
    packed.buffer.fill_(77)
    y, got = lsmgnn.act8(x, "gelu", gated, out=out, packed=packed)
    assert y is out and got is packed and torch.equal(out, want)
    assert torch.equal(got.q, kept.q) and torch.equal(got.scale, kept.scale)
    assert bool((flat[:3] == 9).all()) and bool((flat[3:].view(n, -1)[:, dim:] == 9).all())
    flat, dx = gaps(dim * parts)
    assert lsmgnn.act8_grad(dy, packed, "gelu", gated, dx=dx) is dx and torch.equal(dx, want_dx)
    assert bool((flat[:3] == 9).all()) and bool((flat[3:].view(n, -1)[:, dim * parts:] == 9).all())
    flat, out = gaps(dim * parts)
    full = lsmgnn.pack8(x)
    assert torch.equal(lsmgnn.unpack8(full, out=out), lsmgnn.unpack8(full, dtype))
    assert bool((flat[:3] == 9).all()) and bool((flat[3:].view(n, -1)[:, dim * parts:] == 9).all())


# ------------------------------------------------------------------ captured calls
@pytest.mark.parametrize("n", [900, 30_000])
def test_row_count_and_status_words_of_captured_calls(n):
    """embed_grad_rows_async and the status words of the other calls, replayed with
    indices that are fine and some that name nothing."""
    rng = np.random.default_rng(n)
    num_rows, dim, E = 700, 33, 6
    dy, table = rows(rng, n, dim, torch.float32), rows(rng, num_rows, dim, torch.float32)
    ids = torch.zeros(n, dtype=torch.int64, device="cuda")
    chosen = torch.zeros((n, 2), dtype=torch.int64, device="cuda")
    unique, out = torch.empty_like(ids), torch.empty_like(dy)
    pinned = lsmgnn.PinnedBuffer(16)
    result = pinned.numpy(np.uint64, (2,))
    status = torch.zeros(3, dtype=torch.int64, device="cuda")
    words = [status.data_ptr() + 8 * i for i in range(3)]

    def step():
        lsmgnn.embed_grad_rows_async(dy, ids, num_rows, unique, out, pinned.ptr)
        return (lsmgnn.embed_rows(table, ids, status_ptr=words[0]),
                lsmgnn.embed_grad(dy, ids, num_rows, status_ptr=words[1]),
                lsmgnn.route_plan(chosen, E, status_ptr=words[2]).slot)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for bad in (False, True, False, True):
        new, e = ids_of(rng, n, num_rows), rng.integers(-1, E, (n, 2))
        if bad:
            new[n // 2], e[n - 1, 1] = num_rows, E
        ids.copy_(torch.as_tensor(new).cuda())
        chosen.copy_(torch.as_tensor(e).cuda())
        status.zero_()
        unique.fill_(-5)
        result[:] = 99
        graph.replay()
        torch.cuda.synchronize()
        want_ids, sums, bound = ref.row_sums(ref.f64(dy), new, num_rows, 1.0, None)
        assert result.tolist() == [want_ids.size, lsmgnn.E_RANGE if bad else lsmgnn.OK]
        assert np.array_equal(unique[:want_ids.size].cpu().numpy(), want_ids)
        assert bool((unique[want_ids.size:] == -5).all())
        ref.assert_within(out[:want_ids.size], sums, bound, torch.float32)
        assert status.tolist() == [lsmgnn.E_RANGE if bad else 0] * 3
        assert np.array_equal(ref.f64(got[0]), ref.lookup(ref.f64(table), new, 1.0, None))
        e[e >= E] = -1
        assert np.array_equal(got[2].cpu().numpy(), ref.plan(e, E, 1)[1])
    pinned.close()


# ------------------------------------------------------------------- many experts
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("experts", [65, 300, 1024])
@pytest.mark.parametrize("kind", ["skew", "unordered"])
def test_weight_gradient_of_wider_types_by_many_experts(dtype, experts, kind):
    rng, n = np.random.default_rng(experts), 12_000
    if kind == "skew":
        cut = [0] + np.sort((n * rng.random(experts - 1) ** 5).astype(int)).tolist() + [n]
    else:
        cut = rng.integers(-50, n, experts + 1).tolist()
    check_weight(rng, n, 34, 66, dtype, cut)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_weight_gradient_of_large_tiles_of_wider_types_by_many_experts(dtype):
    rng = np.random.default_rng(8)
    cut = [0] + np.sort((140_000 * rng.random(299) ** 3).astype(int)).tolist() + [140_000]
    check_weight(rng, 140_000, 256, 256, dtype, cut)
