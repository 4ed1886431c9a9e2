"""The 8-bit block format and its product against 64 bits: every byte of the rounding, every result within the bound that its own terms give."""
import numpy as np
import pytest

import block_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mad():
    import torch
    import paper_2106_10860_amd as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def dtype_of(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def data(seed, rows, cols, dtype, special=True):
    """Values over many powers of two, among them exact ties, zeros and whole blocks of zeros."""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 6, (rows, 1)))
    if special:
        x[rng.random((rows, cols)) < 0.05] = 0
        x[rng.random((rows, cols)) < 0.02] *= 30
        x[::7, :128] = 0
        x[1::7] = np.round(x[1::7] * 32) / 32
    return torch.from_numpy(x).to(dtype)


def host(b):
    import torch
    return b.q.view(torch.uint8).cpu().numpy(), b.scale[..., : -(-b.shape[-1] // 128)].cpu().numpy()


def same_bytes(got, want):
    """Equal bytes; any NaN for a NaN."""
    nan = want & 127 == 127
    assert ((got & 127 == 127) == nan).all() and (got[~nan] == want[~nan]).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 129), (3, 16), (17, 128), (128, 128), (129, 255), (200, 510), (33, 1025), (300, 77)])
def test_quantise(mad, rows, cols, dtype):
    print("case quantise", rows, cols, dtype, flush=True)
    x = data(rows * 1000 + cols, rows, cols, dtype_of(dtype))
    xd, x64 = x.cuda(), x.double().numpy()
    for tile in (1, 128):
        want, want_t = ref.quantise(x64, tile), ref.quantise(np.ascontiguousarray(x64.T), tile)
        one, turned, both = (mad.maddness_quantise_blocks(xd, tile, **kw) for kw in ({}, {"transposed": True}, {"both": True}))
        for got, w in ((one, want), (turned, want_t), (both[0], want), (both[1], want_t)):
            q, e = host(got)
            assert (e == w[1]).all()
            same_bytes(q, w[0])
        assert np.array_equal(one.values().double().cpu().numpy(), ref.value(*want, tile))


def test_quantise_strided_and_stacked(mad):
    import torch
    x = data(5, 3 * 140, 301, torch.bfloat16).view(3, 140, 301)
    wide = torch.zeros(3, 150, 333, dtype=torch.bfloat16, device="cuda")
    wide[:, 7:147, 11:312] = x.cuda()
    for tile in (1, 128):
        a, at = mad.maddness_quantise_blocks(wide[:, 7:147, 11:312], tile, both=True)
        want, want_t = ref.quantise(x.double().numpy(), tile), ref.quantise(np.ascontiguousarray(x.double().numpy().transpose(0, 2, 1)), tile)
        for got, w in ((a, want), (at, want_t)):
            q, e = host(got)
            assert (e == w[1]).all()
            same_bytes(q, w[0])


def test_quantise_what_is_not_finite_and_the_ends_of_the_range(mad):
    import torch
    x = data(6, 40, 256, torch.float32, special=False)
    x[0, 3], x[1, 200], x[2, 5] = float("nan"), float("inf"), float("-inf")
    x[3] = float("nan")
    x[4] = 3.4028234663852886e38
    x[5] = 1e-45                                           # a subnormal number: its block's power of two is the least there is
    x[6, 0] = -0.0
    x[7] *= 1e-38
    x[8, :] = 448.0
    x[9, :] = float(np.nextafter(np.float32(448), np.float32(1000)))
    for tile in (1, 128):
        want = ref.quantise(x.double().numpy(), tile)
        q, e = host(mad.maddness_quantise_blocks(x.cuda(), tile))
        assert (e == want[1]).all()
        same_bytes(q, want[0])


@pytest.mark.parametrize("both", [False, True])
def test_quantise_gathered_rows(mad, both):
    import torch
    rng = np.random.default_rng(8)
    T, k, cols, rows = 37, 3, 203, 300
    x = data(9, T, cols, torch.bfloat16)
    factors = torch.from_numpy(rng.standard_normal((T, k)).astype(np.float32))
    source = rng.integers(-3, T * k + 3, rows).astype(np.int32)            # some outside on either side: rows of zeros
    ok = (source >= 0) & (source < T * k)
    at = np.where(ok, source, 0)
    plain = np.where(ok[:, None], x.double().numpy()[at // k], 0)
    for f in (None, factors):
        full = plain if f is None else np.where(ok[:, None], plain.astype(np.float32) * f.numpy().reshape(-1)[at][:, None], 0).astype(np.float64)
        got = mad.maddness_quantise_blocks(x.cuda(), both=both, source=torch.from_numpy(source).cuda(), repeat=k,
                                           factors=None if f is None else f.cuda())
        for g, w in zip(got if both else (got,), (full, np.ascontiguousarray(full.T))):
            want = ref.quantise(w, 1)
            q, e = host(g)
            assert (e == want[1]).all()
            same_bytes(q, want[0])


def bound(A, B, out_dtype):
    """K products, each sum rounded (or cut) to 24 bits, once more to the result's type; where that has 16 bits, the products of a block
    cut off at 2^-11 of the largest, which is at most the product of the two largest factors (twice that, as the cut was measured)."""
    import torch
    K = A.shape[-1]
    terms = np.abs(A) @ np.abs(B).T
    want = A @ B.T
    largest = 0
    if out_dtype is not torch.float32:
        largest = sum(np.outer(np.abs(A[:, k:k + 128]).max(1), np.abs(B[:, k:k + 128]).max(1)) for k in range(0, K, 128))
    unit = {torch.float32: (2.0 ** -24, 2.0 ** -150), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}[out_dtype]
    return want, 2.0 ** -10 * largest + (K + 8) * 2.0 ** -23 * terms * 1.01 + np.abs(want) * unit[0] * 1.01 + unit[1]


def check(got, A, B, label):
    want, tol = bound(A, B, got.dtype)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), f"{label}: {(err > tol).sum()} of {err.size} results off, worst {np.max(err / tol):.2f} of the bound"


SIZES = [(1, 1, 1), (1, 300, 129), (2, 33, 4096), (16, 64, 128), (17, 1000, 510), (64, 250, 1024), (65, 129, 127), (128, 128, 256), (200, 513, 700),
         (257, 260, 2048), (300, 1000, 33), (513, 512, 512), (1000, 770, 384)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("tiles", [(1, 128), (1, 1), (128, 128)])
def test_product(mad, M, N, K, tiles):
    import torch
    print("case product", M, N, K, tiles, flush=True)
    A = mad.maddness_quantise_blocks(data(M + K, M, K, torch.float32).cuda(), tiles[0])
    B = mad.maddness_quantise_blocks(data(N + K + 1, N, K, torch.float32).cuda(), tiles[1])
    a, b = A.values().double().cpu().numpy(), B.values().double().cpu().numpy()
    for dt in (torch.float32, torch.bfloat16, torch.float16):
        got = mad.maddness_block_product(A, B, out_dtype=dt)
        if dt is torch.float16 and np.abs(a @ b.T).max() > 6e4:
            continue
        check(got, a, b, f"{M} x {N} x {K} {tiles} {dt}")
    again = mad.maddness_block_product(A, B, out_dtype=torch.float32)
    assert torch.equal(again, mad.maddness_block_product(A, B, out_dtype=torch.float32))


@pytest.mark.parametrize("M,N,K", [(1, 64, 512), (3, 129, 510), (16, 300, 1000), (17, 300, 1000), (200, 130, 77), (400, 260, 640), (1, 50, 8), (2, 50, 7),
                                   (64, 70, 510), (37, 33, 9), (8, 40, 4000), (1, 40, 20000)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_product_rounds_a_float_operand_as_quantise_does(mad, M, N, K, dtype):
    import torch
    print("case float product", M, N, K, dtype, flush=True)
    wide = torch.zeros(M, K + 5, dtype=dtype_of(dtype), device="cuda")
    wide[:, 3:K + 3] = data(M * N, M, K, dtype_of(dtype)).cuda()
    x = wide[:, 3:K + 3]                                                   # rows at any multiple of an element
    B = mad.maddness_quantise_blocks(data(N, N, K, torch.float32).cuda(), 128)
    got = mad.maddness_block_product(x, B, out_dtype=torch.float32)
    A = mad.maddness_quantise_blocks(x)
    check(got, A.values().double().cpu().numpy(), B.values().double().cpu().numpy(), f"{M} {N} {K}")


def test_product_reads_nothing_beyond_its_columns(mad):
    """NaN bytes and wild exponents right behind the columns, rows of results between others."""
    import torch
    for M, N, K in ((5, 40, 200), (70, 130, 333), (300, 300, 1000)):
        print("case padding", M, N, K, flush=True)
        mats = []
        for rows, tile in ((M, 1), (N, 128)):
            src = mad.maddness_quantise_blocks(data(rows + K, rows, K, torch.float32).cuda(), tile)
            q = torch.full((rows, K // 16 * 16 + 48), 127, dtype=torch.uint8, device="cuda")
            q[:, :K] = src.q.view(torch.uint8)
            blocks = -(-K // 128)
            scale = torch.full((src.scale.shape[0], -(-blocks // 4) * 4 + 4), 255, dtype=torch.uint8, device="cuda")
            scale[:, :blocks] = src.scale[:, :blocks]
            mats.append(mad.BlockMatrix(q.view(torch.float8_e4m3fn)[:, :K], scale, tile))
        out = torch.full((M, N + 7), 5.0, device="cuda")
        mad.maddness_block_product(*mats, out=out[:, 3:N + 3])
        assert (out[:, :3] == 5).all() and (out[:, N + 3:] == 5).all()
        check(out[:, 3:N + 3], *(m.values().double().cpu().numpy() for m in mats), "padding")


def test_product_nan_stays_in_its_row_and_column(mad):
    import torch
    for M, N, K in ((4, 70, 300), (300, 290, 300)):
        x = data(1, M, K, torch.float32, special=False)
        w = data(2, N, K, torch.float32, special=False)
        x[2, 299], w[5, 17] = float("nan"), float("inf")
        got = mad.maddness_block_product(mad.maddness_quantise_blocks(x.cuda()), mad.maddness_quantise_blocks(w.cuda(), 128)).isnan().cpu()
        want = torch.zeros(M, N, dtype=torch.bool)
        want[2], want[:, 5] = True, True
        assert torch.equal(got, want)


def test_product_of_nothing(mad):
    import torch
    A0, B0 = mad.maddness_quantise_blocks(torch.zeros(4, 0, device="cuda")), mad.maddness_quantise_blocks(torch.zeros(9, 0, device="cuda"))
    assert torch.equal(mad.maddness_block_product(A0, B0), torch.zeros(4, 9, dtype=torch.bfloat16, device="cuda"))
    B = mad.maddness_quantise_blocks(torch.ones(9, 32, device="cuda"))
    assert mad.maddness_block_product(torch.zeros(0, 32, device="cuda"), B).shape == (0, 9)


def offsets_of(counts, align):
    return np.concatenate([[0], np.cumsum([-(-c // align) * align for c in counts])]).astype(np.int32)


@pytest.mark.parametrize("counts", [[5], [0, 3, 0, 0, 17, 1, 0], [130, 0, 64, 1, 300, 129], [2] * 70, [1000, 3, 700]])
@pytest.mark.parametrize("N,K", [(96, 200), (300, 512)])
def test_product_by_rows(mad, counts, N, K):
    import torch
    print("case by rows", counts[:6], N, K, flush=True)
    E, off = len(counts), offsets_of(counts, 1)
    S = int(off[-1]) + 9                                                   # rows that nobody has
    A = mad.maddness_quantise_blocks(data(S, S, K, torch.float32).cuda())
    B = mad.maddness_quantise_blocks(data(E, E * N, K, torch.float32).cuda().view(E, N, K), 128)
    out = torch.full((S, N), 7.0, device="cuda")
    mad.maddness_block_product(A, B, torch.from_numpy(off).cuda(), out=out)
    a, b = A.values().double().cpu().numpy(), B.values().double().cpu().numpy()
    for e in range(E):
        if counts[e]:
            check(out[off[e]:off[e + 1]], a[off[e]:off[e + 1]], b[e], f"expert {e}")
    assert (out[off[-1]:] == 7).all()


@pytest.mark.parametrize("T,counts,k", [(4, [3, 0, 2, 5, 0, 1], 3), (50, [20, 0, 17, 1], 2), (300, [130, 0, 64, 1, 300, 129], 3), (2, [1], 1)])
@pytest.mark.parametrize("kind", ["e4m3", "bf16", "f32"])
def test_product_of_gathered_rows(mad, T, counts, k, kind):
    import torch
    print("case gathered", T, counts, kind, flush=True)
    N, K, E, off = 96, 330, len(counts), offsets_of(counts, 4)
    rng = np.random.default_rng(T)
    S = int(off[-1]) + 3
    source = rng.integers(-2, T * k + 2, S).astype(np.int32)              # some rows have none
    x = data(T, T, K, torch.float32 if kind == "e4m3" else dtype_of(kind)).cuda()
    A = mad.maddness_quantise_blocks(x)
    B = mad.maddness_quantise_blocks(data(E, E * N, K, torch.float32).cuda().view(E, N, K), 128)
    out = torch.full((S, N), 7.0, device="cuda")
    mad.maddness_block_product(A if kind == "e4m3" else x, B, torch.from_numpy(off).cuda(), source=torch.from_numpy(source).cuda(), repeat=k, out=out)
    a, b, written = A.values().double().cpu().numpy(), B.values().double().cpu().numpy(), np.zeros(S, bool)
    for e in range(E):
        rows = np.arange(off[e], off[e + 1])
        rows = rows[(source[rows] >= 0) & (source[rows] < T * k)]
        written[rows] = True
        if len(rows):
            check(out[torch.from_numpy(rows).cuda()], a[source[rows] // k], b[e], f"expert {e}")
    assert (out.cpu()[torch.from_numpy(~written)] == 7).all()


@pytest.mark.parametrize("counts", [[128], [0, 3, 0, 200, 129], [1000, 0, 1], [0, 0]])
@pytest.mark.parametrize("M,N", [(40, 70), (300, 260)])
def test_product_by_depth(mad, counts, M, N):
    import torch
    print("case by depth", counts, M, N, flush=True)
    E, off = len(counts), offsets_of(counts, 128)
    S = int(off[-1]) + 50
    A = mad.maddness_quantise_blocks(data(S, M, S, torch.float32).cuda())
    B = mad.maddness_quantise_blocks(data(S + 1, N, S, torch.float32).cuda())
    got = mad.maddness_block_product(A, B, torch.from_numpy(off).cuda(), by="depth", out_dtype=torch.float32)
    a, b = A.values().double().cpu().numpy(), B.values().double().cpu().numpy()
    assert got.shape == (E, M, N)
    for e in range(E):
        if off[e + 1] > off[e]:
            check(got[e], a[:, off[e]:off[e + 1]], b[:, off[e]:off[e + 1]], f"expert {e}")
        else:
            assert (got[e] == 0).all()


def test_product_with_wrong_offsets_stays_in_bounds(mad):
    import torch
    A = mad.maddness_quantise_blocks(torch.ones(100, 256, device="cuda"))
    B = mad.maddness_quantise_blocks(torch.ones(3, 40, 256, device="cuda"), 128)
    for off in ([-5, 50, 20, 1000], [90, 10, 2 ** 31 - 1, -2 ** 31], [0, 0, 0, 0]):
        out = torch.full((100, 40), 3.0, device="cuda")
        mad.maddness_block_product(A, B, torch.tensor(off, dtype=torch.int32, device="cuda"), out=out)
        assert torch.isin(out, torch.tensor([3.0, 256.0], device="cuda")).all()
        got = mad.maddness_block_product(A, mad.maddness_quantise_blocks(torch.ones(40, 256, device="cuda")),
                                         torch.tensor(off, dtype=torch.int32, device="cuda"), by="depth", out_dtype=torch.float32)
        assert torch.isin(got, torch.tensor([0.0, 128.0, 256.0], device="cuda")).all()


def test_gradients_of_a_layer(mad):
    """dX = dY W and dW = dY^T X by the product: against 64 bits on the rounded values, and the gradient of the loss against differences."""
    import torch
    M, N, K = 150, 70, 200
    x, w, dy = data(1, M, K, torch.float32, False), data(2, N, K, torch.float32, False), data(3, M, N, torch.float32, False)
    W, Wt = mad.maddness_quantise_blocks(w.cuda(), 128, both=True)
    assert torch.equal(W.values().T, Wt.values())
    g, gt = mad.maddness_quantise_blocks(dy.cuda(), both=True)
    xt = mad.maddness_quantise_blocks(x.cuda(), transposed=True)
    dx, dw = mad.maddness_block_product(g, Wt, out_dtype=torch.float32), mad.maddness_block_product(gt, xt, out_dtype=torch.float32)
    h = lambda b: b.values().double().cpu().numpy()                        # noqa: E731
    check(dx, h(g), h(W).T, "dx")
    check(dw, h(gt), h(xt), "dw")
    # the loss sum(dY * (X W^T)) along a direction, in 64 bits: the three roundings change it by at most 3 / 16 of the terms' sizes
    v = data(4, M, K, torch.float32, False).double().numpy()
    loss = lambda X: (dy.double().numpy() * (X @ w.double().numpy().T)).sum()      # noqa: E731
    difference = (loss(x.double().numpy() + 1e-3 * v) - loss(x.double().numpy() - 1e-3 * v)) / 2e-3
    terms = (np.abs(v) * (np.abs(dy.double().numpy()) @ np.abs(w.double().numpy()))).sum()
    assert abs((dx.double().cpu().numpy() * v).sum() - difference) <= 3 / 16 * terms


def test_other_stream_and_graph(mad):
    import torch
    A = data(1, 300, 512, torch.bfloat16).cuda()
    B = mad.maddness_quantise_blocks(data(2, 200, 512, torch.float32).cuda(), 128)
    out, small = torch.zeros(300, 200, device="cuda"), torch.zeros(4, 200, device="cuda")
    want, want_small = mad.maddness_block_product(A, B, out_dtype=torch.float32), mad.maddness_block_product(A[:4], B, out_dtype=torch.float32)
    work = torch.empty(300 * 512 + 300 * 4, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    mad.maddness_block_product(A, B, out=out, workspace=work, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            mad.maddness_block_product(A, B, out=out, workspace=work)
            mad.maddness_block_product(A[:4], B, out=small)
    for _ in range(3):
        out.fill_(-1)
        small.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(small, want_small)
        mad.maddness_block_product(A, B)
        torch.cuda.synchronize()


def check_some(got, A, B, label, seed=0):
    """As check, of a few rows and columns, the first and the last ones among them."""
    import torch
    rng = np.random.default_rng(seed)
    rows, cols = (torch.from_numpy(np.unique(np.concatenate([np.arange(min(n, 20)), np.arange(max(n - 20, 0), n), rng.integers(0, n, 100)]))).cuda()
                  for n in got.shape)
    check(got[rows][:, cols], A[rows].double().cpu().numpy(), B[cols].double().cpu().numpy(), label)


def rough(seed, *shape):
    """Rows of very different sizes, made on the device."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 6, (*shape[:-1], 1), generator=g, device="cuda").float())


@pytest.mark.parametrize("M,N,K", [(4100, 4100, 300), (1030, 13100, 5000), (2049, 8200, 4097), (1100, 300, 9000), (3000, 16500, 127)])
def test_product_of_many_rows(mad, M, N, K):
    """Enough for the large tiles; more blocks than exponents are fetched at a time."""
    import torch
    print("case many rows", M, N, K, flush=True)
    A, B = mad.maddness_quantise_blocks(rough(M, M, K)), mad.maddness_quantise_blocks(rough(N, N, K), 128)
    a, b = A.values(), B.values()
    for dt in (torch.float32, torch.bfloat16):
        check_some(mad.maddness_block_product(A, B, out_dtype=dt), a, b, f"{M} x {N} x {K} {dt}")


# lengths that begin at any of the blocks whose exponents are fetched together, and are longer than what is fetched at a time
@pytest.mark.parametrize("counts", [[1024, 4224, 5, 0, 900, 4100, 1, 128, 300, 0, 7, 4096], [1152, 6000, 896, 5000, 1, 2, 3, 4, 5, 6, 7, 8]])
@pytest.mark.parametrize("M,N", [(1030, 1100), (700, 500)])
def test_product_by_depth_of_many_rows(mad, counts, M, N):
    import torch
    print("case by depth, many rows", counts, M, N, flush=True)
    off = offsets_of(counts, 128)
    S = int(off[-1])
    A, B = mad.maddness_quantise_blocks(rough(M, M, S)), mad.maddness_quantise_blocks(rough(N + S, N, S))
    a, b = A.values(), B.values()
    for dt in (torch.float32, torch.bfloat16):
        got = mad.maddness_block_product(A, B, torch.from_numpy(off).cuda(), by="depth", out_dtype=dt)
        for e in range(len(counts)):
            if off[e + 1] > off[e]:
                check_some(got[e], a[:, off[e]:off[e + 1]], b[:, off[e]:off[e + 1]], f"expert {e} {dt}")
            else:
                assert (got[e] == 0).all()


def test_rows_of_a_matrix_without_rows_are_zeros(mad):
    import torch
    x, source = torch.zeros(0, 200, dtype=torch.bfloat16, device="cuda"), torch.full((140,), -1, dtype=torch.int32, device="cuda")
    for factors in (None, torch.zeros(0, device="cuda")):
        for got in mad.maddness_quantise_blocks(x, both=True, source=source, repeat=2, factors=factors):
            assert (got.q.view(torch.uint8) == 0).all() and (got.scale == 127).all()
        assert (mad.maddness_quantise_blocks(x, source=source, repeat=2, factors=factors).q.view(torch.uint8) == 0).all()
    short = mad.maddness_quantise_blocks(torch.zeros(0, 3, device="cuda"), both=True, source=source)
    assert all((b.q.view(torch.uint8) == 0).all() for b in short)


def test_a_source_without_slots(mad):
    import torch
    none, off = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    x = torch.ones(5, 64, device="cuda")
    B = mad.maddness_quantise_blocks(torch.ones(2, 30, 64, device="cuda"), 128)
    assert mad.maddness_block_product(x, B, off, source=none, repeat=2).shape == (0, 30)
    assert mad.maddness_block_product(mad.maddness_quantise_blocks(x), B, off, source=none, repeat=2).shape == (0, 30)
    got = mad.maddness_quantise_blocks(x, both=True, source=none, repeat=2, factors=torch.ones(10, device="cuda"))
    assert got[0].shape == (0, 64) and got[1].shape == (64, 0)


def test_places_beyond_32_bits(mad):
    """More than 2^31 values in each of x, its 8-bit form and the result: the last rows are those of themselves alone."""
    import torch
    rows, cols = (1 << 21) + 100, 1032
    part = rough(3, 4000, cols).to(torch.bfloat16)
    x = part[:1].expand(rows, cols).contiguous()
    x[-4000:] = part
    A, few = mad.maddness_quantise_blocks(x), mad.maddness_quantise_blocks(part)
    assert torch.equal(A.q[-4000:].view(torch.uint8), few.q.view(torch.uint8)) and torch.equal(A.scale[-4000:, :9], few.scale[:, :9])
    turned = mad.maddness_quantise_blocks(x, 128, transposed=True)
    assert torch.equal(turned.q[:, -4000:].view(torch.uint8), mad.maddness_quantise_blocks(x[-4068:], 128, transposed=True).q[:, -4000:].view(torch.uint8))
    del x, turned
    B = mad.maddness_quantise_blocks(rough(4, 1040, cols), 128)
    got = mad.maddness_block_product(A, B)
    check_some(got[-4000:], few.values(), B.values(), "last rows")
    source = torch.arange(rows - 4000, rows, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 4000], dtype=torch.int32, device="cuda")
    B3 = mad.BlockMatrix(B.q.unsqueeze(0), B.scale.unsqueeze(0), 128)
    check_some(mad.maddness_block_product(A, B3, off, source=source), few.values(), B.values(), "gathered last rows")


def test_a_stream_that_is_given_owns_what_the_call_makes(mad):
    """What a call on another stream allocates does not come from the current stream's memory, which that stream may still be using."""
    import torch
    x, side = rough(1, 300, 512), torch.cuda.Stream()
    B = mad.maddness_quantise_blocks(rough(2, 200, 512), 128)
    want = mad.maddness_block_product(x, B)
    free = torch.empty_like(want)
    at = free.data_ptr()
    torch.cuda.synchronize()
    del free                                               # the current stream's, and the first that it would hand out again
    got = mad.maddness_block_product(x, B, stream=side)
    side.synchronize()
    assert got.data_ptr() != at and torch.equal(got, want)
    logits = rough(5, 60, 32)
    ids, weights = mad.maddness_route(logits, 4, stream=side)
    offsets, _, source, place = mad.maddness_order(ids, 32, stream=side)
    y = mad.maddness_combine(got[:40].float(), place, weights, stream=side)
    side.synchronize()
    ids2, weights2 = mad.maddness_route(logits, 4)
    assert torch.equal(ids, ids2) and torch.equal(weights, weights2)
    assert torch.equal(y, mad.maddness_combine(got[:40].float(), mad.maddness_order(ids2, 32)[3], weights2))
