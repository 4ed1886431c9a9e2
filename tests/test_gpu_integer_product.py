"""8-bit integers with a scale for each row, and their product: every number equal to the exact statement's, up to the fp32 roundings of scales, bias and result."""
import numpy as np
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "f16", "bf16"]


@pytest.fixture(params=["native", "python"])
def mad(request, monkeypatch):
    import torch
    import paper_2106_10860_amd as m
    assert torch.cuda.is_available()
    m.lib()
    if request.param == "python":
        monkeypatch.setattr(m, "_native", m._NotBuilt)
    return m


@pytest.fixture(scope="module")
def lib():
    import paper_2106_10860_amd as m
    m.lib()
    return m


def torch_type(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def dev(x, dtype="f32", pad=0, before=0):
    """On the device, with `pad` elements between rows and `before` before the first."""
    import torch
    rows, cols = x.shape
    full = torch.full((before + rows * (cols + pad) + 8,), 77.0, dtype=torch_type(dtype), device="cuda")
    view = full[before:before + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x)))
    return view


def host(t):
    return t.double().cpu().numpy()


def activations(rng, rows, cols):
    x = rng.normal(size=(rows, cols)) * np.exp(rng.normal(size=(rows, 1)))
    x[:, rng.random(cols) < 0.02] *= 20
    return x


def integers(lib, rng, rows, cols, ld=None, junk=True):
    """An IntegerMatrix whose bytes between the columns and the stride are not 0."""
    import torch
    ld = ld or -(-cols // 16) * 16
    q = rng.integers(-127, 128, size=(rows, cols))
    scale = (rng.random(rows) + 0.1).astype(np.float32)
    full = torch.full((rows, ld), 113, dtype=torch.int8, device="cuda")
    full[:, :cols] = torch.from_numpy(q.astype(np.int8)).cuda()
    return lib.IntegerMatrix(full[:, :cols], torch.from_numpy(scale).cuda()), q, scale.astype(np.float64)


def check(got, want, bound, dtype, what=""):
    off = np.abs(host(got) - want)
    most = bound + ref.rounding(np.abs(want) + bound, dtype)
    assert (off <= most).all(), (what, float((off / most).max()), np.unravel_index((off / most).argmax(), off.shape))


# (rows, cols, elements between rows, before the first): below a piece, around pieces and rows of registers, the longest of those and beyond
ROWS = [(1, 1, 0, 0), (3, 2, 1, 1), (5, 7, 0, 3), (4, 8, 0, 0), (9, 9, 1, 1), (2, 63, 0, 0), (130, 510, 0, 0), (5, 512, 3, 1), (7, 513, 0, 1), (6, 1000, 0, 0), (5, 1024, 0, 0),
        (3, 1025, 1, 0), (4, 2048, 0, 0), (3, 2049, 0, 3), (9000, 33, 0, 0), (3, 4096, 0, 0), (2, 4100, 0, 0), (2, 8193, 1, 1), (2, 16384, 0, 0), (2, 16385, 0, 0), (3, 40001, 0, 1)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", ROWS, ids=lambda c: "%dx%d_p%d_o%d" % c)
def test_rows_to_integers(mad, case, dtype):
    rows, cols, pad, before = case
    print("case quantise", case, dtype, flush=True)
    rng = np.random.default_rng(rows * 7 + cols)
    x = activations(rng, rows, cols)
    x_d = dev(x, dtype, pad, before)
    got = mad.maddness_quantise_rows(x_d)
    q, scale = ref.quantise(host(x_d))
    assert got.shape == (rows, cols) and got.q.stride(0) == -(-cols // 16) * 16
    assert np.array_equal(host(got.scale), scale)
    assert np.array_equal(got.q.cpu().numpy().astype(int), q)
    import torch
    padded = torch.as_strided(got.q, (rows, got.q.stride(0)), (got.q.stride(0), 1))
    assert not padded[:, cols:].any()


def test_rows_next_to_borders(mad):
    """Quotients that are exactly halves, and the nearest numbers beside them; the smallest and the largest rows; none; not finite."""
    import torch
    x = np.zeros((12, 260), np.float32)
    x[0, :255] = (np.arange(255) - 127) / 2.0
    x[0, 255] = 127
    for r, scale in ((1, 3.0), (2, np.float32(0.1)), (3, np.float32(7e-5))):
        top = np.float32(127) * np.float32(scale)
        step = np.float32(top / np.float32(127))
        halves = (np.arange(-120, 120, 2) + 0.5).astype(np.float32) * step
        x[r, :120], x[r, 120:240] = halves, np.nextafter(halves, np.float32(0))
        x[r, 250] = top
    x[4, :5] = [1e-45, -1e-45, 3e-45, 1e-44, 0]
    x[5, :4] = [1.17549435e-38 * 60, 1.17549435e-38 * 126.6, -1.17549435e-38, 1e-40]
    x[6, :3] = [3.4028234663852886e38, -3.4e38, 1e30]
    x[8, 17], x[9, 200], x[10, 0] = np.nan, np.inf, -np.inf
    x[8:11, 30] = 5
    x[11, 259] = -1e-3
    got = mad.maddness_quantise_rows(torch.from_numpy(x).cuda())
    q, scale = ref.quantise(x)
    assert np.array_equal(host(got.scale), scale, equal_nan=True) and np.isnan(scale[8:11]).all()
    assert np.array_equal(got.q.cpu().numpy().astype(int), q)
    assert np.abs(q[:8]).max() <= 127


# (M, N, K): single tokens, few rows of every kernel size, edges of tiles, depths below and beyond a block, more tiles than compute units
SIZES = [(1, 1, 1), (1, 5, 16), (1, 300, 130), (2, 17, 127), (7, 33, 128), (16, 64, 129), (17, 31, 255), (1, 200, 4099), (16, 100, 1025), (37, 1000, 510), (63, 65, 600), (64, 129, 256),
         (65, 128, 64), (100, 100, 100), (128, 256, 384), (129, 127, 1000), (257, 300, 77), (300, 513, 2051), (1000, 250, 510), (4097, 4095, 130), (5000, 3000, 33), (3, 40, 131071), (130, 40, 131071)]


@pytest.mark.parametrize("size", SIZES, ids=lambda c: "%dx%dx%d" % c)
def test_integer_product(mad, size):
    M, N, K = size
    print("case product", size, flush=True)
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    import torch
    A, qa, sa = integers(mad, rng, M, K, ld=-(-K // 16) * 16 + 16 * (M % 3))
    B, qb, sb = integers(mad, rng, N, K, ld=-(-K // 16) * 16 + 16 * (N % 2))
    bias = rng.normal(size=N).astype(np.float32) * K
    # whole numbers below 2^53 add exactly in fp64
    exact = (qa.astype(np.float64) @ qb.T.astype(np.float64)) if M * N * K > 1 << 22 else (qa @ qb.T).astype(np.float64)
    v = exact * sa[:, None] * sb[None, :]
    for dtype in DTYPES:
        scale = 1.0 if dtype != "f16" else 1e-4
        A.scale.copy_(torch.from_numpy((sa * scale).astype(np.float32)))
        sa_now = host(A.scale)
        v = exact * sa_now[:, None] * sb[None, :]
        bound = 3.01 * ref.U * np.abs(v) + 2.0 ** -148
        plain = mad.maddness_integer_product(A, B, out_dtype=torch_type(dtype))
        check(plain, v, bound, dtype, (size, dtype))
        with_bias = v + bias * scale
        b = torch.from_numpy(bias * np.float32(scale)).cuda()
        wide = torch.full((M, N + 3), -7.0, dtype=torch_type(dtype), device="cuda")
        got = mad.maddness_integer_product(A, B, bias=b, out=wide[:, 1:N + 1])
        assert got.data_ptr() == wide[:, 1:N + 1].data_ptr()
        want = v + host(b)
        check(got, want, bound + 1.01 * ref.U * (np.abs(want) + bound), dtype, (size, dtype, "bias"))
        assert bool((wide[:, 0] == -7).all()) and bool((wide[:, N + 1:] == -7).all())
        assert np.isfinite(with_bias).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(1, 40, 7), (1, 300, 4096), (3, 65, 8), (8, 100, 4096), (16, 33, 2000), (37, 1000, 510), (64, 64, 512), (64, 70, 520), (65, 64, 100), (200, 300, 1111)],
                         ids=lambda c: "%dx%dx%d" % c)
def test_float_rows_are_rounded_within_the_call(mad, size, dtype):
    """The same to the bit as their rounding and the product of that, whichever kernel rounds them."""
    M, N, K = size
    print("case float rows", size, dtype, flush=True)
    rng = np.random.default_rng(M + N + K)
    x = activations(rng, M, K)
    if M > 2:
        x[1] = 0
    x_d = dev(x, dtype, pad=M % 3, before=M % 2)
    B, qb, sb = integers(mad, rng, N, K)
    import torch
    got = mad.maddness_integer_product(x_d, B, out_dtype=torch.float32)
    A = mad.maddness_quantise_rows(x_d)
    assert torch.equal(got, mad.maddness_integer_product(A, B, out_dtype=torch.float32))
    q, s = ref.quantise(host(x_d))
    want, bound = ref.product(q, s, qb, sb)
    check(got, want, bound, "f32", (size, dtype))
    # a row of no numbers is no numbers, and only it
    x_d[0, 0] = float("nan")
    again = mad.maddness_integer_product(x_d, B, out_dtype=torch.float32)
    assert bool(again[0].isnan().all()) and torch.equal(again[1:], got[1:])


def test_results_do_not_depend_on_other_rows(lib):
    """The sums are exact: whatever kernel the number of rows selects, the same bits, of every form that the products are built in."""
    import torch
    rng = np.random.default_rng(5)
    A, qa, sa = integers(lib, rng, 4200, 1030)
    B, qb, sb = integers(lib, rng, 4096, 1030)
    for dtype in DTYPES:
        bias = torch.from_numpy(rng.normal(size=4096).astype(np.float32) * 1e5).cuda()
        whole = lib.maddness_integer_product(A, B, bias=bias, out_dtype=torch_type(dtype))
        kernels = {lib.maddness_last_kernel()}
        for rows in (1, 16, 32, 64, 65, 500, 1000, 2000, 2300):
            print("case rows", rows, dtype, flush=True)
            part = lib.maddness_integer_product(lib.IntegerMatrix(A.q[:rows], A.scale[:rows]), B, bias=bias, out_dtype=torch_type(dtype))
            kernels.add(lib.maddness_last_kernel())
            assert torch.equal(part, whole[:rows]), rows
        assert len(kernels) == 7, kernels


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_rounded_in_every_form(lib, dtype):
    """Rows that the few-rows kernel rounds by itself, in each of its forms, with a depth that ends inside a piece."""
    import torch
    rng = np.random.default_rng(6)
    B, qb, sb = integers(lib, rng, 4096, 500)
    x_d = dev(activations(rng, 64, 500), dtype, pad=1)
    kernels = set()
    for rows in (1, 16, 32, 33, 64):
        got = lib.maddness_integer_product(x_d[:rows], B, out_dtype=torch.float32)
        kernels.add(lib.maddness_last_kernel())
        q, s = ref.quantise(host(x_d[:rows]))
        want, bound = ref.product(q, s, qb, sb)
        check(got, want, bound, "f32", (rows, dtype))
    assert len(kernels) == 3 and all("integer_few_kernel" in k for k in kernels), kernels


def test_extreme_values(mad):
    """-128, which an integer matrix of the caller's may hold, at the largest depth; empty sizes."""
    import torch
    K = 131071
    q = torch.full((1, K + 1), -128, dtype=torch.int8, device="cuda")[:, :K]
    one = torch.ones(1, device="cuda")
    A = mad.IntegerMatrix(q, one)
    assert mad.maddness_integer_product(A, A, out_dtype=torch.float32).item() == float(K << 14)
    B = mad.IntegerMatrix(torch.zeros((5, 0), dtype=torch.int8, device="cuda"), torch.ones(5, device="cuda"))
    bias = torch.arange(5.0, device="cuda")
    assert torch.equal(mad.maddness_integer_product(torch.zeros((3, 0), device="cuda"), B, bias=bias, out_dtype=torch.float32), bias.expand(3, 5))
    none = mad.maddness_quantise_rows(torch.zeros((0, 32), device="cuda"))
    W = mad.maddness_quantise_rows(torch.ones((4, 32), device="cuda"))
    assert mad.maddness_integer_product(none, W).shape == (0, 4)
    assert mad.maddness_quantise_rows(torch.zeros((3, 0), device="cuda")).scale.tolist() == [1.0] * 3


def test_far_strides(lib):
    """Rows further apart than 32-bit offsets within a tile reach: 130 rows 64 MiB apart span 8.7 GB."""
    import torch
    ld, M, K, N = 1 << 26, 130, 200, 70
    big = torch.empty(M * ld, dtype=torch.int8, device="cuda")
    rng = np.random.default_rng(1)
    q = rng.integers(-127, 128, size=(M, K))
    view = big.as_strided((M, K), (ld, 1))
    view.copy_(torch.from_numpy(q.astype(np.int8)).cuda())
    A = lib.IntegerMatrix(view, torch.ones(M, device="cuda"))
    B, qb, sb = integers(lib, rng, N, K)
    got = lib.maddness_integer_product(A, B, out_dtype=torch.float32)
    want, bound = ref.product(q, np.ones(M), qb, sb)
    check(got, want, bound, "f32")


def test_refusals(mad):
    import torch
    W = mad.maddness_quantise_rows(torch.ones((4, 32), device="cuda"))
    x = torch.ones((3, 32), device="cuda")
    with pytest.raises(TypeError):
        mad.maddness_integer_product(x, x)
    with pytest.raises(TypeError):
        mad.maddness_quantise_rows(x.to(torch.int8))
    with pytest.raises(TypeError):
        mad.maddness_quantise_rows(x.cpu())
    with pytest.raises(ValueError):
        mad.maddness_quantise_rows(x.t())
    with pytest.raises(ValueError):
        mad.maddness_quantise_rows(x[0])
    with pytest.raises(mad.MaddnessError):
        mad.maddness_integer_product(x[:, :16], W)
    with pytest.raises(ValueError):
        mad.maddness_integer_product(x, W, bias=torch.ones(5, device="cuda"))
    with pytest.raises(TypeError):
        mad.maddness_integer_product(x, W, bias=torch.ones(4, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        mad.maddness_integer_product(x, W, out=torch.empty((3, 5), device="cuda"))
    with pytest.raises(ValueError):
        mad.maddness_integer_product(x, W, out=torch.empty((3, 4), device="cuda"), out_dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mad.maddness_integer_product(torch.ones((200, 32), device="cuda"), W, workspace=torch.empty(20000, dtype=torch.uint8, device="cuda")[::2])
    with pytest.raises(mad.MaddnessError):
        mad.maddness_integer_product(torch.ones((200, 32), device="cuda"), W, workspace=torch.empty(100, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_integer_product(x.clone().requires_grad_(), W)
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_quantise_rows(x.clone().requires_grad_())
    q, s = torch.zeros((4, 32), dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    for bad in ((q.float(), s), (q, s.double()), (q.cpu(), s)):
        with pytest.raises(TypeError):
            mad.IntegerMatrix(*bad)
    for bad in ((q[0], s), (q, s[:3]), (q.t(), torch.ones(32, device="cuda")), (q, torch.ones(8, device="cuda")[::2])):
        with pytest.raises(ValueError):
            mad.IntegerMatrix(*bad)
    with pytest.raises(mad.MaddnessError):                         # rows that do not begin at multiples of 16 bytes
        mad.maddness_integer_product(x[:, :20], mad.IntegerMatrix(torch.zeros((4, 20), dtype=torch.int8, device="cuda"), s))


def test_rows_whose_scale_has_no_half(mad):
    """A scale between 2^-126 and 2^-125 with a last bit has a half that is no number of fp32; quotients next to one still go to the nearest integer."""
    import torch
    rng = np.random.default_rng(7)
    x = np.zeros((200, 400), np.float32)
    for row in x:
        row[0] = np.float32(rng.uniform(127 * 2.0 ** -126, 127 * 2.0 ** -125))
        halves = ((np.arange(127) + 0.5) * np.float64(np.float32(row[0] / np.float32(127)))).astype(np.float32)
        near = np.concatenate([halves, np.nextafter(halves, np.float32(0)), np.nextafter(halves, np.float32(1))])
        near[near > row[0]] = 0
        row[1:1 + len(near)] = near * rng.choice([-1, 1], len(near)).astype(np.float32)
    q, scale = ref.quantise(x)
    for wide in (1, 42):                                       # (in registers, and rows that are read again)
        got = mad.maddness_quantise_rows(torch.from_numpy(np.tile(x[:200 // wide], (1, wide))).cuda())
        assert np.array_equal(host(got.scale), scale[:200 // wide])
        assert np.array_equal(got.q.cpu().numpy().astype(int), np.tile(q[:200 // wide], (1, wide)))
    # and within the product
    eye = mad.IntegerMatrix(torch.eye(400, dtype=torch.int8, device="cuda"), torch.ones(400, device="cuda"))
    out = mad.maddness_integer_product(torch.from_numpy(x[:32]).cuda(), eye, out_dtype=torch.float32)
    assert np.array_equal(out.cpu().numpy(), q[:32].astype(np.float32) * scale[:32, None].astype(np.float32))


def test_replaced_tensors_are_checked(mad):
    """A matrix whose values or scales were replaced is refused by the call as by the constructor, on either side, and taken where they fit."""
    import torch
    x = torch.ones((3, 32), device="cuda")
    want = mad.maddness_integer_product(x, mad.maddness_quantise_rows(torch.ones((4, 32), device="cuda")), out_dtype=torch.float32)
    q, s = torch.zeros((4, 32), dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    bad = [("scale", s.half(), TypeError), ("scale", s.double(), TypeError), ("scale", s.cpu(), TypeError), ("scale", None, TypeError), ("scale", s[:3], ValueError), ("scale", s[:1].expand(4), ValueError),
           ("scale", s.reshape(4, 1), ValueError), ("scale", torch.ones(8, device="cuda")[::2], ValueError), ("q", q.float(), TypeError), ("q", q.cpu(), TypeError), ("q", q[0], ValueError),
           ("q", q[:2], ValueError), ("q", q.t(), ValueError), ("q", q[:, :1].expand(4, 32), ValueError), ("q", None, TypeError)]
    for name, value, error in bad:
        for side in (0, 1):
            W = mad.maddness_quantise_rows(torch.ones((4, 32), device="cuda"))
            setattr(W, name, value)
            with pytest.raises(error):
                mad.maddness_integer_product(W if side else x, W)
    W = mad.maddness_quantise_rows(torch.zeros((4, 32), device="cuda"))
    W.q, W.scale = torch.full((4, 32), 127, dtype=torch.int8, device="cuda"), torch.full((4,), 1 / 127, device="cuda")
    assert torch.equal(mad.maddness_integer_product(x, W, out_dtype=torch.float32), want)


@pytest.mark.parametrize("size", [(16384, 1024, 1024), (8192, 1024, 1024), (8192, 1024, 512), (4000, 510, 4096), (300, 1000, 510), (1, 512, 1024)], ids=lambda c: "%dx%dx%d" % c)
def test_bfloat16_rows_to_the_bit(mad, size):
    """Each step of the definition on its own (the quotient's rounding, the exact sum, two products and the result's rounding): the very bits, in tiles of every size.  An
    element of half its row's largest is 63.5 steps, or just below, as the scale's own rounding has it."""
    import torch
    M, N, K = size
    print("case to the bit", size, flush=True)
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x = (torch.randn(M, K, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(M, 1, generator=g, device="cuda"))).bfloat16()
    x[:, 3], x[:, 5] = 16 * x[:, 7], 8 * x[:, 7]
    W = mad.maddness_quantise_rows(torch.randn(N, K, generator=g, device="cuda") / K ** 0.5)
    top = x.double().abs().amax(1, keepdim=True)
    scale = (top / torch.full_like(top, 127.0)).float()        # (a 64-bit quotient is never so near to half an fp32 step that this rounds twice)
    q = torch.round(x.double() / scale.double())
    assert bool((q.abs().amax(1) == 127).all())
    sums = torch.mm(q, W.q.double().T.contiguous())            # (whole numbers below 2^53)
    want = (sums.float() * scale * W.scale).bfloat16()
    assert torch.equal(mad.maddness_integer_product(x, W), want)
    assert torch.equal(mad.maddness_integer_product(mad.maddness_quantise_rows(x), W), want)
