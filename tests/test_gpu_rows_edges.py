"""The operators on trained rows at the ends of their ranges, against 64-bit
references on the GPU."""
import numpy as np
import pytest

from tests import rows_reference as ref
from tests.test_gpu_embed import TYPES, rows

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from paper_2407_15264_amd import lsmgnn  # noqa: E402

LEAST = 2.0 ** -149  # a float32's spacing next to 0: a product rounded once more where it is subnormal


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lsmgnn.lib()


def dev(a, dtype=torch.float32):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.float64).to(dtype).cuda()


# --------------------------------------- gated activations of numbers far apart
A_FAR = [-1e30, -1000.0, -400.0, -300.0, -200.0, -104.0, -90.0, -87.0, -50.0, -10.0, -3.0, -1.0, -0.25, 0.0, 0.5, 1.0]
SIZES = [1e38, 1e36, 1e25, 1e20, 1e10, 1.0, 1e-10, 1e-30]


def far_rows(dtype, rng, n, most):
    """(a, b, dy) of every combination of A_FAR and SIZES, and n drawn ones, of sizes up
    to 10^most, as the type holds them."""
    sizes = [v for v in SIZES if v <= 10.0 ** most]
    small = [v for v in A_FAR if abs(v) <= 10.0 ** most]
    a, b, g = (v.reshape(-1) for v in np.meshgrid(small, sizes + [-v for v in sizes], sizes, indexing="ij"))
    sign = lambda: rng.choice([-1.0, 1.0], n)  # noqa: E731
    a = np.concatenate([a, -10.0 ** rng.uniform(-2, 2.8, n)])
    b = np.concatenate([b, sign() * 10.0 ** rng.uniform(-37, most, n)])
    g = np.concatenate([g, sign() * 10.0 ** rng.uniform(-37, most, n)])
    return [ref.f64(dev(v, dtype)).reshape(-1, 1) for v in (a, b, g)]


def check_far(dtype, act, forward, slope, most=38):
    a, b, g = far_rows(dtype, np.random.default_rng(1), 4000, most)
    ka, kb = ref.pack(a)[2], ref.pack(b)[2]
    f, bf = forward(a)
    kf, bkf = forward(ka)
    kdf, bdf = slope(ka)
    fits = np.abs(np.stack([f * b, g * kb * kdf, g * kf])).max(0)[:, 0] < 3e38
    a, b, g, kb, f, bf, kf, bkf, kdf, bdf = (v[fits] for v in (a, b, g, kb, f, bf, kf, bkf, kdf, bdf))
    assert a.shape[0] > 3000
    y, p = lsmgnn.act8(dev(np.concatenate([a, b], 1), dtype), act, True)
    ref.assert_within(y, f * b, (bf + 2 * ref.U32 * np.abs(f)) * np.abs(b) + LEAST, dtype, "y")
    dx = lsmgnn.act8_grad(dev(g, dtype), p, act, True)
    ref.assert_within(dx[:, :1], g * kb * kdf, np.abs(g * kb) * (bdf + 3 * ref.U32 * np.abs(kdf)) + LEAST, dtype,
                      "da")
    ref.assert_within(dx[:, 1:], g * kf, np.abs(g) * (bkf + 2 * ref.U32 * np.abs(kf)) + LEAST, dtype, "db")
    # without a gate
    _, p = lsmgnn.act8(dev(a, dtype), act)
    fits = np.abs(g * kdf)[:, 0] < 3e38
    dx = lsmgnn.act8_grad(dev(g, dtype), p, act)
    ref.assert_within(dx[torch.as_tensor(fits).cuda()], (g * kdf)[fits],
                      (np.abs(g) * (bdf + 2 * ref.U32 * np.abs(kdf)) + LEAST)[fits], dtype, "dx")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_silu_with_large_and_small_factors(dtype):
    """Finite inputs with finite results: none of the products on the way leaves
    the range of a float."""
    check_far(dtype, "silu", lambda x: ref.act("silu", x)[:2], lambda x: ref.act("silu", x)[2:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activation_of_infinities(dtype, act):
    """f(inf) = inf; f(-inf) is what the formula is there, NaN."""
    x = torch.tensor([[float("inf")], [-float("inf")], [float("nan")], [1.0]], device="cuda").to(dtype)
    y = lsmgnn.act8(x, act)[0].cpu()
    assert y[0, 0] == float("inf") and torch.isnan(y[1:3]).all() and torch.isfinite(y[3, 0])
    for b in (2.0, -2.0):
        gate = torch.full_like(x, b)
        y = lsmgnn.act8(torch.cat([x, gate], 1), act, True)[0].cpu()
        assert y[0, 0] == b * float("inf") and torch.isnan(y[1:3]).all() and torch.isfinite(y[3, 0])
    # an infinite gate of an ordinary value
    y = lsmgnn.act8(torch.tensor([[-3.0, float("inf")], [-1000.0, float("inf")], [2.0, -float("inf")]],
                                 device="cuda").to(dtype), act, True)[0].cpu()
    assert (y == -float("inf")).all()


# ----------------------------------------------------------- gelu's negative tail
def gelu64(x, dtype):
    """f and its bound, 16 units of 2^-24 of itself: e 2^n to 4 of them (the exponent's
    parts, exp2), the scaled tail to 10, two products; in 16 bits the rounding of the
    exponent x^2 / 2 too."""
    f = x * 0.5 * torch.special.erfc(torch.as_tensor(-x / np.sqrt(2))).numpy()
    return f, (16 + (0 if dtype == torch.float32 else 1) * x * x / 2) * ref.U32 * np.abs(f)


def gelu_slope64(x, dtype):
    """f' and its bound, as many units of what is added up."""
    cdf = 0.5 * torch.special.erfc(torch.as_tensor(-x / np.sqrt(2))).numpy()
    pdf = np.exp(-0.5 * x * x) / np.sqrt(2 * np.pi)
    units = 16 + (0 if dtype == torch.float32 else 1) * x * x / 2
    return cdf + x * pdf, units * ref.U32 * (cdf + np.abs(x) * pdf)


@pytest.mark.parametrize("dtype", TYPES)
def test_gelu_tail(dtype):
    """Every value down to where 32 bits hold none, and its slope, as good relatively
    as it is near 0."""
    x = np.concatenate([np.linspace(-14, 6, 20001), [-13.9, -5.5, -5.0, 12.0, 30.0, 1000.0, -20.0, -1000.0]])
    x = ref.f64(dev(x, dtype)).reshape(-1, 1)
    y, p = lsmgnn.act8(dev(x, dtype), "gelu")
    f, bf = gelu64(x, dtype)
    ref.assert_within(y, f, bf + LEAST, dtype, "y")
    kept = ref.pack(x)[2]
    df, bdf = gelu_slope64(kept, dtype)
    dx = lsmgnn.act8_grad(torch.ones_like(y), p, "gelu")
    ref.assert_within(dx, df, bdf + LEAST, dtype, "dx")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gelu_with_large_and_small_factors(dtype):
    check_far(dtype, "gelu", lambda x: gelu64(x, dtype), lambda x: gelu_slope64(x, dtype))


# ------------------------------------------------- values kept as a power too large
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_of_the_largest_numbers(dtype, act):
    """The largest numbers are kept as 2^128, which 32 bits hold as an infinity only;
    their gradients are those of 2^128 all the same."""
    big = torch.finfo(dtype).max
    x = torch.tensor([[big, 0.5], [-big, 0.5], [1.0, big], [1.0, -big], [-3.0, big]], device="cuda").to(dtype)
    dy = torch.full((5, 1), 0.25, device="cuda").to(dtype)
    both = ref.pack(ref.f64(x).reshape(-1, 1))[2].reshape(5, 2)
    a, b, g = both[:, :1], both[:, 1:], ref.f64(dy)
    assert np.abs(both).max() == 2.0 ** 128
    _, p = lsmgnn.act8(x, act, True)
    f, df = (v.numpy() for v in f64_of(act, torch.as_tensor(a)))
    dx = lsmgnn.act8_grad(dy, p, act, True)
    # 20 units of 2^-24: 16 for f and f', 2^128 as the float below it, the products
    want = np.concatenate([g * b * df, g * f], 1)
    ref.assert_within(dx, want, 20 * ref.U32 * (np.abs(want) + np.concatenate([np.abs(g * b), 0 * g], 1)), dtype)
    _, p = lsmgnn.act8(x[:2, :1].contiguous(), act)
    ref.assert_within(lsmgnn.act8_grad(dy[:2], p, act), (g * df)[:2], 20 * ref.U32, dtype)


def f64_of(act, x):
    """f and f' in 64 bits where x may be very large."""
    if act == "silu":
        p, q = torch.sigmoid(x), torch.sigmoid(-x)
        return x * p, p * (1 + x * q)
    cdf = 0.5 * torch.special.erfc(-x / 2 ** 0.5)
    return x * cdf, cdf + x * torch.exp(-0.5 * x * x) / (2 * np.pi) ** 0.5


# --------------------------------------------------- the weight gradient's row of dy
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ld", [0, 1, 70])
def test_weight_gradient_of_one_row_whatever_its_stride(dtype, ld):
    """A single row has no next one: its stride says nothing, and no element of dy
    counts twice."""
    dout = 70
    x = torch.tensor([[0.5, -0.25, 1.0, 0.125, -0.5]], device="cuda").to(dtype)
    dy = torch.ones((1, dout), device="cuda").to(dtype)
    dy[0, 3], dy[0, 40] = float("inf"), -float("inf")
    p = lsmgnn.pack8(x)
    dw = torch.empty((5, dout), device="cuda")
    code = lsmgnn.ELEMENT_TYPES[ref.name_of(dtype)]
    rc = lsmgnn.lib().lsmgnn_weight_grad8(p.q.data_ptr(), p.scale.data_ptr(), 1, 5, dy.data_ptr(), dout, ld, code, None,
                                          1, dw.data_ptr(), 0, None, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == lsmgnn.OK
    assert np.array_equal(ref.f64(dw), ref.f64(x).T * ref.f64(dy))


@pytest.mark.parametrize("power", [-60, -90, -100, -105, -110, -115, -120, -126, -130])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weight_gradient_of_small_numbers(dtype, power):
    """A float32 dy is three bfloat16 numbers, whose least is 2^-133: its elements count
    to within that."""
    rng = np.random.default_rng(-power)
    x = rng.integers(-100, 101, (200, 8)).astype(np.float64)
    x[:, 0] = 127
    dy = rng.standard_normal((200, 6)) * 2.0 ** power
    x, dy = dev(x, torch.float32), dev(dy, dtype)
    p = lsmgnn.pack8(x)
    v, g = ref.f64(lsmgnn.unpack8(p, torch.float32)), ref.f64(dy)
    got = lsmgnn.weight_grad8(p, dy)[0]
    size = np.abs(v).T @ (np.abs(g) * 202 * ref.U32 + (2.0 ** -133 if dtype == torch.float32 else 0.0))
    ref.assert_within(got, v.T @ g, size, torch.float32)


# ----------------------------------------------------- more lanes than one launch has
def room_for(gigabytes):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GiB of device memory")


def test_kept_rows_of_one_value():
    """More than 2^30 rows of one value each; whole numbers are kept exactly."""
    room_for(40)
    n = (1 << 30) + 77
    x = torch.randint(-64, 65, (n, 1), dtype=torch.int8, device="cuda").to(torch.bfloat16)
    p = lsmgnn.pack8(x)
    assert torch.equal(lsmgnn.unpack8(p), x)
    del p
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    _, p = lsmgnn.act8(x, "silu", out=y)
    assert torch.equal(lsmgnn.unpack8(p), x)
    lsmgnn.act8_grad(x, p, "silu", dx=dx)
    del p
    for a in range(0, n, 1 << 27):  # every row was written
        assert not torch.isnan(y[a:a + (1 << 27)]).any() and not torch.isnan(dx[a:a + (1 << 27)]).any()
    for a in (0, (1 << 28) - 500, (1 << 29) - 500, (1 << 30) - 500, n - 1000):
        part = x[a:a + 1000]
        want, kept = lsmgnn.act8(part, "silu")
        assert torch.equal(y[a:a + 1000], want)
        assert torch.equal(dx[a:a + 1000], lsmgnn.act8_grad(part, kept, "silu"))


def test_combine_gradient_of_many_tokens():
    """33 pieces of a row take 64 lanes: 2^32 of them and the unused rows' too."""
    room_for(100)
    n, dim = (1 << 33) // 129, 129
    dy = torch.randint(-100, 100, (n, dim), dtype=torch.int8, device="cuda").float()
    slot = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    source = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    dz = torch.empty((n, dim), device="cuda")
    rc = lsmgnn.lib().lsmgnn_route_combine_grad(dy.data_ptr(), n, dim, dim, 0, None, dim, slot.data_ptr(),
                                                source.data_ptr(), None, 1, n, dz.data_ptr(), dim, None,
                                                torch.cuda.current_stream().cuda_stream)
    assert rc == lsmgnn.OK
    for a in range(0, n, 1 << 23):
        b = min(n, a + (1 << 23))
        assert torch.equal(dz[n - b:n - a].flip(0), dy[a:b])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_factors_that_are_only_small(dtype, act):
    """Where no factor of a wave is above 2^40 they are multiplied as they are."""
    if act == "silu":
        check_far(dtype, "silu", lambda x: ref.act("silu", x)[:2], lambda x: ref.act("silu", x)[2:], 11)
    else:
        check_far(dtype, "gelu", lambda x: gelu64(x, dtype), lambda x: gelu_slope64(x, dtype), 11)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_a_large_neighbour_changes_nothing(dtype, act):
    """A row's results are the same bits whether or not one beside it takes its wave
    the large numbers' way."""
    rng = np.random.default_rng(3)
    x, dy = rows(rng, 64, 96, dtype), rows(rng, 64, 48, dtype)
    y, p = lsmgnn.act8(x, act, True)
    dx = lsmgnn.act8_grad(dy, p, act, True)
    far = x.clone()
    far[::3, 60] = torch.finfo(dtype).max / 4
    y_far, p_far = lsmgnn.act8(far, act, True)
    dx_far = lsmgnn.act8_grad(dy, p_far, act, True)
    same = torch.arange(64, device="cuda") % 3 != 0
    assert torch.equal(y_far[same], y[same]) and torch.equal(dx_far[same], dx[same])


@pytest.mark.parametrize("n", [0, 5, 13_000])
def test_gradient_of_more_than_one_launch_clears(n):
    """A whole gradient of 65 GiB: no row keeps what was there."""
    room_for(80)
    num_rows, dim = 33_300_000, 1024
    grad = torch.ones((num_rows, dim), dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(n, device="cuda") * 2500 + 7
    dy = torch.full((n, dim), 2.0, dtype=torch.bfloat16, device="cuda")
    lsmgnn.embed_grad(dy, ids, num_rows, grad=grad)
    assert bool((grad[ids] == 2).all())
    grad[ids] = 0
    for a in range(0, num_rows, 4_000_000):
        assert not grad[a:a + 4_000_000].any()
