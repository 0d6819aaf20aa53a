"""GPU parity of rows in four-bit numbers and of their products: codes and scales bit for bit, products of the very values within the sums' roundings."""
import numpy as np
import pytest

from oracle import experts as ox
from test_gpu_experts import HALF, STEP32, counts_of, near, offsets_of, wide

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ms():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2508_12801_amd as m
    m.load_library()
    return m


def bits_equal(ms, x):
    q, scales = ms.mxfp4_quantise(x)
    codes, want = ox.mxfp4_quantise(wide(x))
    assert np.array_equal(scales.cpu().numpy(), want)
    ok = np.repeat(want != 255, 32, axis=-1)
    assert np.array_equal(ox.mxfp4_unpack(q.cpu().numpy())[ok], codes[ok])
    values = ox.mxfp4_values(codes, want)
    for dtype in (torch.bfloat16, torch.float32):
        got = ms.mxfp4_dequantise(q, scales, dtype=dtype)
        assert got.dtype == dtype and got.shape == x.shape
        assert np.array_equal(wide(got), values, equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(1, 32), (7, 64), (3, 5, 96), (130, 160), (2, 2080), (33, 32)])
def test_quantise(ms, shape, dtype):
    print(f"quantise {shape} {dtype}", flush=True)
    rng = np.random.default_rng(shape[-1])
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-20, 20, (*shape[:-1], 1))
    bits_equal(ms, torch.from_numpy(x.astype(np.float32)).cuda().to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantise_ties_ends_and_odd_values(ms, dtype):
    print(f"quantise ends {dtype}", flush=True)
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 7.0, 7.9375])
    rows = []
    eps = {torch.bfloat16: 2.0 ** -7, torch.float32: 2.0 ** -23}[dtype]
    for e in (-140, -133, -128, -127, -126, -125, -124, -100, -3, 0, 5, 100, 124):
        for v in (grid, grid * (1 + eps), grid * (1 - eps)):
            b = np.concatenate([v, -v])
            b[0] = 4.0                                   # the block's power of two is 2^e
            rows.append(np.ldexp(b, e))
    rows += [np.zeros(32), np.full(32, -0.0), np.eye(1, 32, 5)[0] * 2.0 ** -126, np.full(32, 3.0e38), np.eye(1, 32, 31)[0] * 1e-45]
    for bad in (np.inf, -np.inf, np.nan):
        rows.append(np.where(np.arange(32) == 17, bad, 1.0))
    with np.errstate(over="ignore"):
        x = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda().to(dtype)
    bits_equal(ms, x)


def test_quantise_from_any_address(ms):
    print("quantise misaligned", flush=True)
    for dtype in (torch.bfloat16, torch.float32):
        flat = torch.randn(1 + 5 * 64, device="cuda").to(dtype)
        bits_equal(ms, flat[1:].view(5, 64))
        q = torch.empty(1 + 5 * 32, dtype=torch.uint8, device="cuda")[1:].view(5, 32)
        s = torch.empty(1 + 5 * 2, dtype=torch.uint8, device="cuda")[1:].view(5, 2)
        ms.mxfp4_quantise(flat[1:].view(5, 64), out=(q, s))
        a, b = ms.mxfp4_quantise(flat[1:].view(5, 64).clone())
        assert torch.equal(q, a) and torch.equal(s, b)
        x = torch.empty(1 + 5 * 64, dtype=dtype, device="cuda")[1:].view(5, 64)
        assert torch.equal(ms.mxfp4_dequantise(q, s, out=x), ms.mxfp4_dequantise(a, b, dtype=dtype))


def four_bits(rng, shape, spread=6):
    """Random codes (every one of the sixteen) and scales, on the device, and their values."""
    codes = rng.integers(0, 16, shape).astype(np.uint8)
    scales = (127 + rng.integers(-spread, spread, (*shape[:-1], shape[-1] // 32))).astype(np.uint8)
    return torch.from_numpy(ox.mxfp4_pack(codes)).cuda(), torch.from_numpy(scales).cuda(), ox.mxfp4_values(codes, scales)


SHAPES = [(3, 5, 64, 64), (1, 1, 32, 8), (2, 1, 32, 1), (4, 33, 96, 40), (3, 130, 288, 136), (5, 64, 256, 256), (2, 300, 512, 264), (3, 17, 160, 35),
          (2, 129, 1056, 127), (3, 257, 64, 250), (8, 16, 320, 96), (2, 520, 768, 520), (130, 3, 32, 16), (3, 40, 2080, 24), (2, 31, 224, 500)]


@pytest.mark.parametrize("kind", ["some", "full", "empty"])
@pytest.mark.parametrize("E,C,K,N", SHAPES)
def test_products_in_four_bits(ms, E, C, K, N, kind):
    print(f"mxfp4 products E={E} C={C} K={K} N={N} {kind}", flush=True)
    rng = np.random.default_rng(E + C + K + N)
    counts = counts_of(kind, E, C, rng)
    off, off_h = offsets_of(counts)
    xq, xs, xr = four_bits(rng, (E, C, K))
    for j, n in enumerate(counts):
        xs[j, n:] = 255                                     # NaN behind the rows
    wq, ws, wr = four_bits(rng, (E, N, K))
    y, size = ox.expert_matmul(xr, wr, off_h, transposed=True)
    near(ms.expert_matmul_mxfp4(xq, xs, wq, ws, off), y, HALF["bf16"] * np.abs(y) + (K + 1) * STEP32 * size)
    # gates of a size at which the unit bends
    wq, ws, wr = four_bits(rng, (E, 2 * N, K))
    scale = int(np.round(np.log2(np.sqrt((xr ** 2).mean() * (wr ** 2).mean() * K))))
    ws, wr = (ws.int() - scale).to(torch.uint8), wr * 2.0 ** -scale
    gu, size = ox.expert_matmul(xr, wr, off_h, transposed=True)
    sums = (K + 1) * STEP32 * size
    h, silu = ox.swiglu(gu), np.abs(gu[..., :N] * ox.sigmoid(gu[..., :N]))
    bound = HALF["bf16"] * np.abs(h) + 1.1 * sums[..., :N] * (np.abs(gu[..., N:]) + sums[..., N:]) + silu * sums[..., N:] + 8 * STEP32 * np.abs(h)
    near(ms.expert_swiglu_mxfp4(xq, xs, wq, ws, off), h, bound)


def test_products_in_four_bits_from_any_address(ms):
    print("mxfp4 misaligned", flush=True)
    rng = np.random.default_rng(6)
    E, C, K, N = 2, 40, 96, 24
    off, off_h = offsets_of([40, 11])
    xq, xs, xr = four_bits(rng, (E, C, K))
    wq, ws, wr = four_bits(rng, (E, N, K))
    want = ms.expert_matmul_mxfp4(xq, xs, wq, ws, off)

    def moved(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    for i in range(4):
        args = [moved(a) if n == i else a for n, a in enumerate((xq, xs, wq, ws))]
        assert torch.equal(ms.expert_matmul_mxfp4(*args, off), want)


def test_a_scale_of_255_is_a_nan_in_its_row(ms):
    print("mxfp4 nan", flush=True)
    rng = np.random.default_rng(7)
    off, _ = offsets_of([40])
    xq, xs, _ = four_bits(rng, (1, 40, 96))
    wq, ws, _ = four_bits(rng, (1, 24, 96))
    clean = ms.expert_matmul_mxfp4(xq, xs, wq, ws, off)
    xs[0, 5, 2] = 255
    got = ms.expert_matmul_mxfp4(xq, xs, wq, ws, off)
    assert torch.isnan(got[0, 5]).all()
    got[0, 5] = clean[0, 5]
    assert torch.equal(got, clean)


def test_a_serving_layer_in_four_bits(ms):
    """Rows quantised once per token, dispatched as they are, through both products and back: against 64 bits on the same four-bit values."""
    print("mxfp4 layer", flush=True)
    rng = np.random.default_rng(8)
    T, d, E, k, n, C = 96, 128, 8, 2, 64, 30
    x = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).cuda().to(torch.bfloat16)
    W = torch.from_numpy((rng.standard_normal((d, E)) / 11).astype(np.float32)).cuda().to(torch.bfloat16)
    r = ms.route_xw(x, W, None, k, C)
    off = r["expert_offsets"]
    q, s = ms.mxfp4_quantise(x)
    xq = ms.dispatch_tokens(q.view(torch.bfloat16), off, r["disp_token"], E, C).view(torch.uint8)
    xs = ms.dispatch_tokens(s.view(torch.bfloat16), off, r["disp_token"], E, C).view(torch.uint8)
    whole = ms.mxfp4_quantise(ms.dispatch_tokens(x, off, r["disp_token"], E, C))
    assert torch.equal(xq, whole[0]) and torch.equal(xs, whole[1])
    wi = ms.mxfp4_quantise(torch.from_numpy((rng.standard_normal((E, 2 * n, d)) / 11).astype(np.float32)).cuda())
    wo = ms.mxfp4_quantise(torch.from_numpy((rng.standard_normal((E, d, n)) / 8).astype(np.float32)).cuda())
    h = ms.expert_swiglu_mxfp4(xq, xs, *wi, off)
    hq = ms.mxfp4_quantise(h)
    out = ms.expert_matmul_mxfp4(*hq, *wo, off)
    y = ms.combine(out, r["assign"], r["token_pos"], r["gates"])
    values = lambda t: ox.mxfp4_values(ox.mxfp4_unpack(t[0].cpu().numpy()), t[1].cpu().numpy())     # noqa: E731
    off_h = off.cpu().numpy()
    gu, size = ox.expert_matmul(values((xq, xs)), values(wi), off_h, True)
    want = ox.swiglu(gu)
    # a rounding to bf16, and sums of 128 exact products of some tens in magnitude
    assert np.abs(wide(h) - want).max() <= (HALF["bf16"] + 1e-4) * np.abs(want).max()
    want, size = ox.expert_matmul(values(hq), values(wo), off_h, True)
    near(out, want, HALF["bf16"] * np.abs(want) + 65 * STEP32 * size)
    import oracle
    want = oracle.combine(wide(out), r["assign"].cpu().numpy(), r["token_pos"].cpu().numpy(), wide(r["gates"]))
    near(y, want, 1e-6 * np.abs(want).max())
