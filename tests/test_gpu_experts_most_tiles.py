"""GPU parity of the gated unit at the most tiles of its widest kernel, sampled against products in 64 bits; tolerances as in test_gpu_experts."""
import pytest

from test_gpu_experts import HALF, STEP32
from test_gpu_experts_tiles import ms, within  # noqa: F401  (ms: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("C", [64, 65])
def test_gated_unit_of_the_most_tiles(ms, C):
    """1024 experts, 2^20 gates each: with 65 rows the most tiles of 256 x 128 that a card's memory has room for, more than one launch counts threads for."""
    print(f"most tiles C={C}", flush=True)
    E, K, N = 1024, 8, 1 << 20
    if torch.cuda.mem_get_info()[0] < (190 << 30):
        torch.cuda.empty_cache()
        if torch.cuda.mem_get_info()[0] < (190 << 30):
            pytest.skip("too little memory free")
    gen = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn(E, C, K, generator=gen, device="cuda").bfloat16()
    w = torch.empty(E, K, 2 * N, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    off = (torch.arange(E + 1, device="cuda") * C).int()
    off[8:] -= C                                               # expert 7 has no row
    h = ms.expert_swiglu(x, w, off)["h"]
    columns = torch.cat([torch.arange(300), torch.arange(N // 2 - 150, N // 2 + 150), torch.arange(N - 300, N)]).cuda()
    for j in (0, 6, 7, 8, 127, 128, 255, 256, 511, 512, 513, 1000, 1022, 1023):
        y, size = (a @ b for a, b in ((x[j].double(), w[j][:, torch.cat([columns, columns + N])].double()),
                                      (x[j].double().abs(), w[j][:, torch.cat([columns, columns + N])].double().abs())))
        if j == 7:
            y, size = torch.zeros_like(y), torch.zeros_like(size)
        size = size * ((K + 1) * STEP32)
        n = columns.numel()
        g, u, eg, eu = y[:, :n], y[:, n:], size[:, :n], size[:, n:]
        silu = g * torch.sigmoid(g)
        want = u * silu
        within(h[j][:, columns], want, HALF["bf16"] * want.abs() + 1.1 * eg * (u.abs() + eu) + silu.abs() * eu + 8 * STEP32 * want.abs())
    del h, w
    torch.cuda.empty_cache()
