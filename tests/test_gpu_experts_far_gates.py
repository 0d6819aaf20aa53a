"""GPU parity of the gated unit and its gradient where e^-g leaves fp32 (g below -88.7) and where u and dh are so large that what they are multiplied by
still counts: against the same in 64 bits.

Tolerances.  The sums here are exact (one or a few products of powers of two and short numbers).  The sigmoid is within two and a half steps of fp32 (the
exponential a step, its sum with one half a step, the reciprocal a step), the unit has two products more, its gradient a difference, a sum and two products:
within eight steps of the result, as gates lie beyond 4 on either side of zero, where nothing in 1 + g (1 - s) cancels.  Rounding the result adds half a step of
its type, below the normal numbers half of the smallest one."""
import pytest

from oracle import experts as ox
from test_gpu_experts import HALF, STEP32, torch_type
from test_gpu_experts_tiles import ms, within  # noqa: F401  (ms: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LEAST = {"bf16": 2.0 ** -133, "fp32": 2.0 ** -148}       # smallest numbers, or two of them: a product's and its factors'


def gates(n, dtype):
    """n gates: from -190 to -4, closely from -105 to -79, and from 4 to 100."""
    a, b, c = n // 4, n // 2, n - n // 4 - n // 2
    g = torch.cat([torch.linspace(-190, -4, a, dtype=torch.float64), torch.linspace(-105, -79, b, dtype=torch.float64),
                   torch.linspace(4, 100, c, dtype=torch.float64)])
    return g.to(torch_type(dtype)).cuda()


def unit(g, u):
    return u * (g * torch.from_numpy(ox.sigmoid(g.cpu().numpy())).cuda())


def near(got, want, dtype):
    assert bool(torch.isfinite(want.to(torch_type(dtype))).all())        # nothing here leaves the type
    within(got, want, (HALF[dtype] + 8 * STEP32) * want.abs() + LEAST[dtype])


# few tiles, tiles of 64 rows, 128 x 128, 256 x 256 of bf16, rows that begin anywhere
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("E,C,K,N", [(1, 3, 8, 200), (6, 60, 16, 600), (6, 60, 16, 601), (16, 300, 8, 1000), (64, 270, 8, 264), (3, 700, 9, 131)])
def test_gated_unit(ms, E, C, K, N, transposed, dtype):
    print(f"far gates E={E} C={C} K={K} N={N} {dtype} transposed={transposed}", flush=True)
    g = gates(N, dtype)
    exponents = torch.tensor([0, 20, 60, 100, 118, -30], device="cuda").repeat((E + 5) // 6)[:E]
    u = torch.exp2(exponents.double())
    x = torch.zeros(E, C, K, device="cuda", dtype=g.dtype)
    x[:, :, 0] = x[:, :, 1] = 1.0
    w = torch.zeros(E, K, 2 * N, device="cuda", dtype=g.dtype)
    w[:, 0, :N], w[:, 1, N:] = g, u[:, None].to(g.dtype)
    off = (torch.arange(E + 1, device="cuda") * C).int()
    weight = w.transpose(1, 2).contiguous() if transposed else w
    want = unit(g.double()[None, None, :], u[:, None, None]).expand(E, C, N)
    near(ms.expert_swiglu(x, weight, off, transposed=transposed)["h"], want, dtype)
    r = ms.expert_swiglu(x, weight, off, transposed=transposed, want_gate_up=True)
    near(r["h"], want, dtype)
    assert torch.equal(r["gate_up"], torch.cat([g.expand(E, C, N), u[:, None, None].to(g.dtype).expand(E, C, N)], dim=2))


@pytest.mark.parametrize("E,C,N", [(2, 7, 24), (6, 70, 264), (64, 270, 264)])
def test_gated_unit_of_four_bits(ms, E, C, N):
    print(f"far gates mxfp4 E={E} C={C} N={N}", flush=True)
    K = 128
    x = torch.zeros(E, C, K, device="cuda")
    x[:, :, :4] = 1.0
    # gates of up to three numbers with one power of two: -64, -72, ... -192
    parts = torch.tensor([(0, 64, 0), (64, 8, 0), (64, 16, 0), (64, 24, 0), (96, 0, 0), (96, 8, 0), (96, 16, 0), (96, 32, 0), (96, 48, 0), (96, 64, 32)], dtype=torch.float32)
    w = torch.zeros(E, 2 * N, K, device="cuda")
    w[:, :N, 1:4] = -parts.repeat((N + 9) // 10, 1)[:N].cuda()
    u = torch.exp2(torch.tensor([0, 20, 60, 100, 118, -30], device="cuda").repeat((E + 5) // 6)[:E].float())
    w[:, N:, 0] = u[:, None]
    off = (torch.arange(E + 1, device="cuda") * C).int()
    got = ms.expert_swiglu_mxfp4(*ms.mxfp4_quantise(x), *ms.mxfp4_quantise(w), off)
    want = unit(w[:, None, :N, 1:4].double().sum(-1), u.double()[:, None, None]).expand(E, C, N)
    near(got, want, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [128, 131, 512])
def test_gradient(ms, N, dtype):
    print(f"far gates gradient N={N} {dtype}", flush=True)
    g = gates(N, dtype)
    down = g < 0
    rows_u, rows_d = [], []
    # large, and one large and one small whose product or partial products leave fp32 while the result does not
    for eu, ed in ((0, 0), (60, 60), (110, 110), (120, 60), (60, 120), (125, -40), (-40, 125), (-100, 120), (120, -100)):
        u, d = torch.full_like(g, 2.0 ** eu), torch.full_like(g, -2.0 ** ed)
        if eu + ed > 110:                                  # gates above zero take it whole
            u, d = torch.where(down, u, torch.ones_like(u)), torch.where(down, d, torch.ones_like(d))
        for a, b in ((u, d), (-u, -d)):
            rows_u.append(a), rows_d.append(b)
    u, d = torch.stack(rows_u), torch.stack(rows_d)
    C = u.shape[0]
    gd, ud, dd = g.double().expand(C, N), u.double(), d.double()
    s, t = (torch.from_numpy(ox.sigmoid(a.cpu().numpy())).cuda() for a in (gd, -gd))
    dg, du, h = dd * ud * s * (1 + gd * t), dd * gd * s, ud * gd * s
    fits = torch.stack([a.abs() < 2.0 ** 120 for a in (dg, du, h)]).all(0)
    # what leaves the type is none of this: such gates get factors of one
    u, d = torch.where(fits, u, torch.ones_like(u)), torch.where(fits, d, torch.ones_like(d))
    ud, dd = u.double(), d.double()
    dg, du, h = dd * ud * s * (1 + gd * t), dd * gd * s, ud * gd * s
    gate_up = torch.cat([g.expand(C, N), u], dim=1).reshape(1, C, 2 * N).contiguous()
    got = ms.expert_swiglu_backward(gate_up, d.reshape(1, C, N).contiguous(), torch.tensor([0, C], dtype=torch.int32, device="cuda"))
    near(got["h"][0], h, dtype)
    near(got["dgate_up"][0, :, N:], du, dtype)
    near(got["dgate_up"][0, :, :N], dg, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N", [64, 67])
def test_what_stands_beside_them(ms, N, dtype):
    """Far gates, large products and NaN change no bit of the values beside them; a NaN stays one, and a gate of minus infinity shuts."""
    print(f"beside far gates N={N} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(N)
    draw = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch_type(dtype))       # noqa: E731
    C = 6
    gate_up, dh, off = draw(1, C, 2 * N), draw(1, C, N), torch.tensor([0, C], dtype=torch.int32, device="cuda")
    clean = ms.expert_swiglu_backward(gate_up, dh, off)
    odd, big = gate_up.clone(), dh.clone()
    for row, at, gate, up, d in ((0, 3, -95.0, 1.0, 1.0), (1, 10, 1.0, 2.0 ** 100, 2.0 ** 60), (2, 33, float("nan"), 1.0, 1.0), (3, N - 1, -float("inf"), 1.0, 1.0),
                                 (4, N - 2, -300.0, 2.0 ** 100, -2.0 ** 100), (5, 0, 0.5, float("inf"), 1.0)):
        odd[0, row, at], odd[0, row, N + at], big[0, row, at] = gate, up, d
    got = ms.expert_swiglu_backward(odd, big, off)
    hit = ((odd != gate_up)[..., :N] | (odd != gate_up)[..., N:] | (big != dh))
    assert int(hit.sum()) == 6
    assert torch.equal(got["h"][~hit], clean["h"][~hit])
    for half in (slice(0, N), slice(N, 2 * N)):
        assert torch.equal(got["dgate_up"][..., half][~hit], clean["dgate_up"][..., half][~hit])
    for a in (got["h"], got["dgate_up"][..., :N], got["dgate_up"][..., N:]):
        assert torch.isnan(a[0, 2, 33]) and a[0, 3, N - 1] == 0
    assert got["h"][0, 5, 0] == float("inf") and torch.isinf(got["dgate_up"][0, 5, 0]) and torch.isfinite(got["dgate_up"][0, 5, N])
    # the products' own epilogue: one expert's gates by one input column, its ups by another
    x = torch.zeros(1, 1, 8, device="cuda", dtype=odd.dtype)
    x[0, 0, :2] = 1.0
    w = torch.zeros(1, 8, 2 * N, device="cuda", dtype=odd.dtype)
    w[0, 0, :N], w[0, 1, N:] = gate_up[0, 0, :N], gate_up[0, 0, N:]
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    clean = ms.expert_swiglu(x, w, one)["h"]
    w[0, 0, 5], w[0, 0, N - 1] = float("nan"), -95.0
    h = ms.expert_swiglu(x, w, one)["h"]
    assert torch.isnan(h[0, 0, 5])
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[5] = rest[N - 1] = False
    assert torch.equal(h[0, 0, rest], clean[0, 0, rest])
