"""GPU parity of the experts' products where there are too few tiles for the compute units and four wavefronts share each one's slabs, at the numbers of
tiles at which that begins and ends, and of the kernels behind it; against products in 64 bits on the GPU.  Tolerances as in test_gpu_experts: (K + 1) steps
of fp32 of the sum of the products' magnitudes, in whichever order they are added, and the rounding of the result."""
import pytest

from test_gpu_experts import HALF, STEP32, torch_type
from test_gpu_experts_tiles import check_forward, check_four_bits, ms, ragged, within  # noqa: F401  (ms: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def operands(E, C, K, N, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, off, keep = ragged(E, C, gen)
    t = torch_type(dtype)
    nan = torch.full((), float("nan"), device="cuda", dtype=t)
    x = torch.where(keep, torch.randn(E, C, K, generator=gen, device="cuda").to(t), nan)
    w = (torch.randn(E, K, N, generator=gen, device="cuda") * 2 * K ** -0.5).to(t)
    return off, keep, x, w, nan, gen


# one slab to more than are on their way at once, whole and not
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K", [1, 4, 8, 31, 32, 64, 72, 128, 160, 192, 201, 256, 320, 328, 384, 392, 448, 513, 1032])
def test_forward_of_few_rows_at_every_number_of_slabs(ms, K, gated, transposed, dtype):
    print(f"few tiles K={K} {dtype} gated={gated} transposed={transposed}", flush=True)
    for E, C, N in ((5, 37, 136), (8, 64, 1000 if gated else 2000)):         # tiles of 32 rows and of 64
        off, keep, x, w, _, _ = operands(E, C, K, 2 * N if gated else N, dtype, K)
        check_forward(ms, x, w, off, keep, dtype, K, gated, transposed)


# tiles of 32 x 64 and of 64 x 64 at 256, 512, 1024 and 2048 of them and one more column of tiles (8, or, of rows that begin anywhere, 3 columns of the
# result more), with what comes behind: 64 x 128 in six stages and three, 64 x 256, 32 x 128, 128 x 128
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("more", [0, 8, 3])
@pytest.mark.parametrize("E,C,N", [(8, 17, 2048), (16, 32, 2048), (1, 1, 16384), (8, 33, 2048), (8, 64, 2048), (8, 128, 2048), (16, 200, 1024), (16, 256, 1024),
                                   (32, 200, 1024)])
def test_forward_at_the_limits(ms, E, C, N, more, dtype):
    for gated in (False, True):
        for transposed in (False, True):
            print(f"limits E={E} C={C} N={N} more={more} {dtype} gated={gated} transposed={transposed}", flush=True)
            columns = N // 2 + more if gated else N + more
            K = 200 if more != 3 else 203
            off, keep, x, w, _, _ = operands(E, C, K, 2 * columns if gated else columns, dtype, E + C + more)
            check_forward(ms, x, w, off, keep, dtype, K, gated, transposed)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("E,C,K,N", [(1, 1, 1, 1), (2, 1000, 512, 1024), (3, 333, 200, 136), (5, 64, 37, 41), (1, 513, 1024, 2048), (1, 300, 1024, 2056), (4, 65, 33, 1000),
                                     (4, 200, 1027, 961), (4, 130, 1089, 1027), (16, 70, 392, 392), (16, 129, 521, 700)])
def test_weight_gradient(ms, E, C, K, N, dtype):
    print(f"few tiles wgrad E={E} C={C} K={K} N={N} {dtype}", flush=True)
    off, keep, x, _, nan, gen = operands(E, C, K, 1, dtype, C + N)
    dy = torch.where(keep, torch.randn(E, C, N, generator=gen, device="cuda").to(x.dtype), nan)
    xd, dyd = torch.where(keep, x.double(), 0.0).transpose(1, 2).contiguous(), torch.where(keep, dy.double(), 0.0)
    want, size = xd @ dyd, xd.abs() @ dyd.abs()
    outs = (torch.float32, torch.bfloat16) if dtype == "bf16" else (torch.float32,)
    for out in outs:
        within(ms.expert_matmul_wgrad(x, dy, off, dtype=out), want,
               HALF["bf16" if out == torch.bfloat16 else "fp32"] * want.abs() + (C + 1) * STEP32 * size)


# from eight slabs of 256 on; tiles of 32, of 64 and, one more column of them, the kernels behind
@pytest.mark.parametrize("K", [2016, 2048, 2080, 2304, 4128])
@pytest.mark.parametrize("E,C,N", [(3, 37, 136), (8, 60, 1024), (8, 60, 2048), (8, 60, 2056), (2, 500, 1000)])
def test_four_bits(ms, E, C, N, K):
    print(f"few tiles four bits E={E} C={C} K={K} N={N}", flush=True)
    check_four_bits(ms, E, C, K, N, K + C)


def test_rows_do_not_depend_on_what_the_others_hold(ms):
    """The joined sums are those of a row alone: the same bits whichever rows stand beside it, and at every call."""
    off, keep, x, w, _, gen = operands(6, 40, 456, 264, "bf16", 3)
    first = ms.expert_matmul(x, w, off)
    other = x.clone()
    other[:, 1::2] = torch.randn(other[:, 1::2].shape, generator=gen, device="cuda").bfloat16()
    again = ms.expert_matmul(other, w, off)
    assert torch.equal(first[:, ::2], again[:, ::2])
    for _ in range(20):
        assert torch.equal(ms.expert_matmul(x, w, off), first)


@pytest.mark.parametrize("gated", [False, True])
def test_the_most_experts_with_the_widest_rows(ms, gated):
    """1024 experts' one row to 2^20 columns: more tiles than one launch counts threads for.  One product to a sum: one rounding."""
    print(f"widest rows gated={gated}", flush=True)
    E, N = 1024, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(E, 1, 1, generator=gen, device="cuda").bfloat16()
    w = torch.empty(E, 1, 2 * N if gated else N, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    off = torch.arange(E + 1, device="cuda").int()
    off[8:] -= 1                                               # expert 7 has no row
    got = ms.expert_swiglu(x, w, off)["h"] if gated else ms.expert_matmul(x, w, off)
    for j in (0, 6, 7, 8, 255, 256, 511, 512, 513, 1000, 1022, 1023):
        y = x[j].double() * w[j].double()
        if j == 7:
            y = torch.zeros_like(y)
        if gated:
            g, u = y[:, :N], y[:, N:]
            y = u * (g * torch.sigmoid(g))
        within(got[j], y, HALF["bf16"] * y.abs() * (1 + 16 * STEP32) + (8 * STEP32 * y.abs() if gated else 0.0) + 2.0 ** -133)
