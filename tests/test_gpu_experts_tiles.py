"""GPU parity of the experts' products at the sizes at which another kernel, tile or number of slabs takes them, against products in 64 bits on the GPU.
Tolerances as in test_gpu_experts: (K + 1) steps of fp32 of the sum of the products' magnitudes, and the rounding of the result."""
import numpy as np
import pytest

from oracle import experts as ox
from test_gpu_experts import HALF, STEP32, torch_type

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ms():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2508_12801_amd as m
    m.load_library()
    return m


def ragged(E, C, gen):
    """Rows per expert: none, one, all but one, all, and anything between."""
    n = torch.randint(0, C + 1, (E,), generator=gen, device="cuda")
    n[:4] = torch.tensor([C, 0, 1, C - 1], device="cuda")[:E]
    off = torch.cat([n.new_zeros(1), n.cumsum(0)]).int()
    return n, off, (torch.arange(C, device="cuda")[None, :] < n[:, None])[..., None]


def within(got, want, bound):
    assert got.shape == want.shape
    bad = ~((got.double() - want).abs() <= bound)            # NaN is not within
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist())


def check_forward(ms, x, w, off, keep, dtype, K, gated, transposed):
    weight = w.transpose(1, 2).contiguous() if transposed else w
    xd, wd = torch.where(keep, x.double(), 0.0), w.double()
    y, size = xd @ wd, (xd.abs() @ wd.abs()) * ((K + 1) * STEP32)
    if not gated:
        within(ms.expert_matmul(x, weight, off, transposed=transposed), y, HALF[dtype] * y.abs() + size)
        return
    r = ms.expert_swiglu(x, weight, off, transposed=transposed, want_gate_up=True)
    within(r["gate_up"], y, HALF[dtype] * y.abs() + size)
    N = y.shape[-1] // 2
    g, u, eg, eu = y[..., :N], y[..., N:], size[..., :N], size[..., N:]
    silu = g * torch.sigmoid(g)
    h = u * silu
    within(r["h"], h, HALF[dtype] * h.abs() + 1.1 * eg * (u.abs() + eu) + silu.abs() * eu + 8 * STEP32 * h.abs())
    assert torch.equal(ms.expert_swiglu(x, weight, off, transposed=transposed)["h"], r["h"])


# 256 tiles of 256 x 256 and more: one to nine slabs of 64, whole and not, the last rows and columns in a tile of their own
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K", [8, 64, 72, 128, 136, 192, 256, 320, 376, 384, 448, 520, 576])
def test_forward_in_many_large_tiles(ms, K, gated, transposed):
    print(f"large tiles K={K} gated={gated} transposed={transposed}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(K)
    E, C, N = 64, 270, 264
    n, off, keep = ragged(E, C, gen)
    x = torch.randn(E, C, K, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(E, K, 2 * N if gated else N, generator=gen, device="cuda") * 2 * K ** -0.5).bfloat16()
    x = torch.where(keep, x, torch.full_like(x, float("nan")))
    check_forward(ms, x, w, off, keep, "bf16", K, gated, transposed)


@pytest.mark.parametrize("C", [1, 63, 64, 65, 127, 128, 200, 256, 300, 448, 513])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_weight_gradient_in_many_large_tiles(ms, C, out):
    print(f"large tiles wgrad C={C} {out}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(C)
    E, K, N = 64, 264, 520
    n, off, keep = ragged(E, C, gen) if C > 1 else (None, torch.arange(E + 1, device="cuda").int(), torch.ones(E, 1, 1, dtype=torch.bool, device="cuda"))
    nan = torch.full((), float("nan"), device="cuda", dtype=torch.bfloat16)
    x = torch.where(keep, torch.randn(E, C, K, generator=gen, device="cuda").bfloat16(), nan)
    dy = torch.where(keep, torch.randn(E, C, N, generator=gen, device="cuda").bfloat16(), nan)
    xd, dyd = torch.where(keep, x.double(), 0.0).transpose(1, 2).contiguous(), torch.where(keep, dy.double(), 0.0)
    want, size = xd @ dyd, xd.abs() @ dyd.abs()
    within(ms.expert_matmul_wgrad(x, dy, off, dtype=out), want, (HALF["bf16"] if out == torch.bfloat16 else HALF["fp32"]) * want.abs() + (C + 1) * STEP32 * size)


# tiles of 64 rows: up to 256 of them, up to 512, more (and rows of 512 bytes of W); one block of 32 rows for fp32; 128 x 128
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("E,C,K,N,dtype", [(8, 64, 456, 520, "bf16"), (64, 33, 200, 600, "bf16"), (64, 64, 328, 1160, "bf16"), (96, 7, 64, 1096, "bf16"),
                                           (8, 64, 456, 520, "fp32"), (64, 70, 100, 600, "fp32"), (64, 32, 132, 520, "fp32"), (40, 5, 68, 1028, "fp32"),
                                           (16, 200, 264, 136, "bf16"), (16, 200, 264, 136, "fp32")])
def test_forward_in_small_tiles(ms, E, C, K, N, dtype, gated, transposed):
    print(f"small tiles E={E} C={C} K={K} N={N} {dtype} gated={gated} transposed={transposed}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(C + K)
    n, off, keep = ragged(E, C, gen)
    t = torch_type(dtype)
    x = torch.randn(E, C, K, generator=gen, device="cuda").to(t)
    w = (torch.randn(E, K, 2 * N if gated else N, generator=gen, device="cuda") * 2 * K ** -0.5).to(t)
    x = torch.where(keep, x, torch.full_like(x, float("nan")))
    check_forward(ms, x, w, off, keep, dtype, K, gated, transposed)


def four_bits(ms, gen, *shape):
    """Rows in four bits and their values (exact in fp32)."""
    x = torch.randn(*shape, generator=gen, device="cuda") * torch.exp2(torch.randint(-2, 3, (*shape[:-1], 1), generator=gen, device="cuda").float())
    q = ms.mxfp4_quantise(x)
    return q, ms.mxfp4_dequantise(*q, dtype=torch.float32).double()


def check_four_bits(ms, E, C, K, N, seed, moved=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, off, keep = ragged(E, C, gen)
    (xq, xs), xd = four_bits(ms, gen, E, C, K)
    xs = torch.where(keep, xs, torch.full_like(xs, 255))
    xd = torch.where(keep, xd, 0.0)
    for gated in (False, True):
        (wq, ws), wd = four_bits(ms, gen, E, 2 * N if gated else N, K)
        ws, wd = ws - 5, wd / 32                              # gates of a size at which the unit bends
        if moved:                                             # scales that begin one byte off
            flat = torch.empty(ws.numel() + 1, dtype=torch.uint8, device="cuda")
            flat[1:] = ws.reshape(-1)
            ws = flat[1:].view(ws.shape)
        wt = wd.transpose(1, 2).contiguous()
        y, size = xd @ wt, (xd.abs() @ wt.abs()) * ((K + 1) * STEP32)
        if not gated:
            within(ms.expert_matmul_mxfp4(xq, xs, wq, ws, off), y, HALF["bf16"] * y.abs() + size)
            continue
        g, u, eg, eu = y[..., :N], y[..., N:], size[..., :N], size[..., N:]
        silu = g * torch.sigmoid(g)
        h = u * silu
        within(ms.expert_swiglu_mxfp4(xq, xs, wq, ws, off), h, HALF["bf16"] * h.abs() + 1.1 * eg * (u.abs() + eu) + silu.abs() * eu + 8 * STEP32 * h.abs())


# slabs of 256; scales of rows that begin on 4 bytes (K a multiple of 128) and that do not
@pytest.mark.parametrize("K", [32, 128, 256, 384, 512, 640, 768, 896, 1024, 1056, 1152, 1280, 1408, 1568, 2048])
def test_four_bits_in_many_large_tiles(ms, K):
    print(f"large tiles mxfp4 K={K}", flush=True)
    check_four_bits(ms, 64, 270, K, 264, K)


@pytest.mark.parametrize("E,C,K,N", [(8, 64, 480, 520), (64, 40, 704, 264), (16, 200, 608, 136), (3, 300, 1024, 40)])
def test_four_bits_in_small_tiles(ms, E, C, K, N):
    print(f"small tiles mxfp4 E={E} C={C} K={K} N={N}", flush=True)
    check_four_bits(ms, E, C, K, N, K)


def test_four_bits_with_scales_off_four_bytes(ms):
    print("large tiles mxfp4, scales one byte off", flush=True)
    check_four_bits(ms, 64, 270, 512, 264, 3, moved=True)


def test_results_that_go_past_the_last_cache(ms):
    """256 MiB of them behind few slabs: forward, gated, four bits; sampled experts, and zeros behind every expert's rows."""
    print("large results", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    E, C, K, N = 64, 2048, 256, 1032
    n, off, keep = ragged(E, C, gen)
    x = torch.randn(E, C, K, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(E, K, N, generator=gen, device="cuda") / 8).bfloat16()
    y = ms.expert_matmul(x, w, off)
    r = ms.expert_swiglu(x, torch.cat([w, w.flip(1)], dim=2).contiguous(), off, want_gate_up=True)
    xq, wq = ms.mxfp4_quantise(x), ms.mxfp4_quantise(w.transpose(1, 2).contiguous())
    yq = ms.expert_matmul_mxfp4(*xq, *wq, off)
    for out in (y, r["h"], r["gate_up"], yq):
        assert not bool((out != 0).logical_and(~keep).any())
    xv, wv = (ms.mxfp4_dequantise(*a, dtype=torch.float32) for a in (xq, wq))
    for j in (0, 3, 17, 63):
        k = int(n[j])
        for got, a, b in ((y, x[j, :k], w[j]), (yq, xv[j, :k], wv[j].T), (r["gate_up"][..., :N], x[j, :k], w[j]), (r["gate_up"][..., N:], x[j, :k], w[j].flip(0))):
            a, b = a.double(), b.double().contiguous()
            want = a @ b
            within(got[j, :k], want, HALF["bf16"] * want.abs() + (K + 1) * STEP32 * (a.abs() @ b.abs()))


def test_every_row_of_one_expert(ms):
    """All tokens with one of many experts, and a single expert of long rows."""
    print("one expert has all", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for E, C, K, N, full in ((64, 1100, 128, 264, 37), (1, 4100, 512, 4104, 0)):
        x = torch.randn(E, C, K, generator=gen, device="cuda").bfloat16()
        w = (torch.randn(E, K, N, generator=gen, device="cuda") * K ** -0.5).bfloat16()
        n = torch.zeros(E, dtype=torch.int64, device="cuda")
        n[full] = C
        off = torch.cat([n.new_zeros(1), n.cumsum(0)]).int()
        y = ms.expert_matmul(x, w, off)
        want = x[full].double() @ w[full].double()
        within(y[full], want, HALF["bf16"] * want.abs() + (K + 1) * STEP32 * (x[full].double().abs() @ w[full].double().abs()))
        assert int((y != 0).any(dim=2).any(dim=1).sum()) == 1
        dw = ms.expert_matmul_wgrad(x, y, off)
        want = x[full].double().T.contiguous() @ y[full].double()
        within(dw[full], want, HALF["fp32"] * want.abs() + (C + 1) * STEP32 * (x[full].double().abs().T.contiguous() @ y[full].double().abs()))


def test_the_oracle_agrees_with_the_products_above():
    """The 64-bit products used here against the oracle's, on one small case."""
    rng = np.random.default_rng(0)
    x, w = rng.normal(size=(3, 4, 5)), rng.normal(size=(3, 5, 6))
    y, _ = ox.expert_matmul(x, w, np.array([0, 4, 8, 12]))
    assert np.allclose((torch.from_numpy(x) @ torch.from_numpy(w)).numpy(), y)
