"""GPU parity around the experts where results are too large for the last cache (256 MiB) and leave past it, and of the tiles that only many rows which
begin anywhere reach.  Sampled experts against products in 64 bits on the GPU; tolerances as in test_gpu_experts."""
import pytest

from test_gpu_experts import HALF, STEP32, torch_type
from test_gpu_experts_tiles import four_bits, ms, ragged, within  # noqa: F401  (ms: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def check_weight_gradient(ms, E, C, K, N, dtype, outs, experts):
    gen = torch.Generator(device="cuda").manual_seed(C + N)
    n, off, keep = ragged(E, C, gen)
    nan = torch.full((), float("nan"), device="cuda", dtype=torch_type(dtype))
    x = torch.where(keep, torch.randn(E, C, K, generator=gen, device="cuda").to(nan.dtype), nan)
    dy = torch.where(keep, torch.randn(E, C, N, generator=gen, device="cuda").to(nan.dtype), nan)
    for out in outs:
        got = ms.expert_matmul_wgrad(x, dy, off, dtype=out)
        assert got.dtype == out and got.numel() * got.element_size() >= (256 << 20 if C > 100 else 0)
        for j in experts:
            r = int(n[j])
            a, b = x[j, :r].double().T.contiguous(), dy[j, :r].double()
            want, size = a @ b, a.abs() @ b.abs()
            within(got[j], want, HALF["bf16" if out == torch.bfloat16 else "fp32"] * want.abs() + (r + 1) * STEP32 * size)
        assert not bool(got[1].any())                       # an expert without rows


# 256 x 256 tiles of bf16 and 128 x 128 of fp32, an even number of slabs and an odd one that ends early; the last tiles whole and not
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("C,K,N", [(256, 2048, 1024), (200, 2056, 1032)])
def test_weight_gradient(ms, C, K, N, dtype):
    print(f"large dW C={C} K={K} N={N} {dtype}", flush=True)
    outs = (torch.float32, torch.bfloat16) if dtype == "bf16" else (torch.float32,)
    check_weight_gradient(ms, 64, C, K, N, dtype, outs, (0, 2, 3, 31, 63))


@pytest.mark.parametrize("dtype,E,C,K,N", [("fp32", 8, 40, 1089, 1027), ("bf16", 8, 40, 1089, 1027), ("fp32", 12, 70, 1027, 1091)])
def test_weight_gradient_of_rows_that_begin_anywhere(ms, dtype, E, C, K, N):
    print(f"many tiles of odd rows E={E} C={C} K={K} N={N} {dtype}", flush=True)
    check_weight_gradient(ms, E, C, K, N, dtype, (torch.float32,), range(E))


# scales that do not begin on four bytes: 128 x 128; that do: 256 x 256
@pytest.mark.parametrize("K", [288, 384])
def test_four_bits(ms, K):
    print(f"large four-bit results K={K}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(K)
    E, C, N = 64, 2048, 1032
    n, off, keep = ragged(E, C, gen)
    (xq, xs), xd = four_bits(ms, gen, E, C, K)
    xs = torch.where(keep, xs, torch.full_like(xs, 255))
    for gated in (False, True):
        (wq, ws), wd = four_bits(ms, gen, E, 2 * N if gated else N, K)
        ws, wd = ws - 5, wd / 32
        got = ms.expert_swiglu_mxfp4(xq, xs, wq, ws, off) if gated else ms.expert_matmul_mxfp4(xq, xs, wq, ws, off)
        assert got.numel() * 2 >= 256 << 20 and not bool((got != 0).logical_and(~keep).any())
        for j in (0, 2, 3, 40, 63):
            r = int(n[j])
            a, b = xd[j, :r], wd[j].T.contiguous()
            y, size = a @ b, (a.abs() @ b.abs()) * ((K + 1) * STEP32)
            if not gated:
                within(got[j, :r], y, HALF["bf16"] * y.abs() + size)
                continue
            g, u, eg, eu = y[:, :N], y[:, N:], size[:, :N], size[:, N:]
            silu = g * torch.sigmoid(g)
            h = u * silu
            within(got[j, :r], h, HALF["bf16"] * h.abs() + 1.1 * eg * (u.abs() + eu) + silu.abs() * eu + 8 * STEP32 * h.abs())


@pytest.mark.parametrize("dtype,T,d,C", [("bf16", 20000, 2048, 5200), ("fp32", 9000, 2048, 2600), ("bf16", 20000, 2056, 5200)])
def test_combine_backward(ms, dtype, T, d, C):
    """Rows in and out of 256 MiB and more: every slot, and every place that holds nothing."""
    print(f"large combine backward T={T} d={d} C={C} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(T + d)
    E, k = 16, 4
    assign = torch.rand(T, E, generator=gen, device="cuda").argsort(1)[:, :k].int()
    assign[torch.rand(T, k, generator=gen, device="cuda") < 0.1] = -1
    chosen = torch.zeros(T, E + 1, dtype=torch.int32, device="cuda").scatter_(1, torch.where(assign < 0, E, assign).long(), 1)[:, :E]
    counts = chosen.sum(0)
    assert int(counts.max()) <= C
    pos = (chosen.cumsum(0).int() - 1).gather(1, assign.clamp(min=0).long()).int()
    off = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    keep = (torch.arange(C, device="cuda")[None, :] < counts[:, None])[..., None]
    t = torch_type(dtype)
    eo = torch.where(keep, torch.randn(E, C, d, generator=gen, device="cuda").to(t), torch.full((), float("nan"), device="cuda", dtype=t))
    assert eo.numel() * eo.element_size() >= 256 << 20
    dy, gate = torch.randn(T, d, generator=gen, device="cuda"), torch.randn(T, k, generator=gen, device="cuda")
    out = dict(dexpert_out=torch.full_like(eo, 7.0), dgates=torch.full_like(gate, 7.0))
    got = ms.combine_backward(dy, eo, assign, pos, gate, off, out=out)
    assert not bool((got["dexpert_out"] != 0).logical_and(~keep).any())
    for s in range(k):
        i = torch.nonzero(assign[:, s] >= 0)[:, 0]
        e, p, g = assign[i, s].long(), pos[i, s].long(), dy[i].double()
        want = gate[i, s].double()[:, None] * g
        within(got["dexpert_out"][e, p], want, (HALF[dtype] + HALF["fp32"]) * (1 + HALF["fp32"]) * want.abs())
        rows = eo[e, p].double()
        dot, size = (rows * g).sum(1), (rows * g).abs().sum(1)
        within(got["dgates"][i, s], dot, HALF["fp32"] * dot.abs() + (d + 1) * STEP32 * size)
        assert not bool(got["dgates"][assign[:, s] < 0, s].any())
