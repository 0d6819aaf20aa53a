"""GPU parity of the experts' products, the gated unit, their gradients and combine's gradient against the 64-bit oracle.

Tolerances.  A product of two bf16 or of two four-bit numbers is exact in fp32; a product of fp32 numbers and every addition is off by at most a step
of fp32, 2^-23 of its result (half a step where it is rounded to nearest), so a sum of K products is within (K + 1) 2^-23 of the sum of the products'
magnitudes.  Rounding the result to bf16 adds 2^-8 of it, to fp32 2^-24."""
import numpy as np
import pytest

import oracle
from oracle import experts as ox

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
STEP32 = 2.0 ** -23


@pytest.fixture(scope="module")
def ms():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2508_12801_amd as m
    m.load_library()
    return m


def torch_type(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def normal(rng, shape, dtype, scale=1.0):
    """(device tensor, its values in 64 bits)."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).cuda().to(torch_type(dtype))
    return t, t.double().cpu().numpy()


def wide(t):
    return t.double().cpu().numpy()


def counts_of(kind, E, C, rng):
    if kind == "full":
        return np.full(E, C)
    if kind == "empty":
        return np.zeros(E, dtype=int)
    n = rng.integers(0, C + 1, E)
    n[0], n[-1] = C, 0
    if E > 2:
        n[1] = 1
    return n


def offsets_of(counts):
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return torch.from_numpy(off).cuda(), off


def spoil(t, counts):
    """What lies behind an expert's rows is nobody's business: NaN and infinities there change nothing."""
    for j, n in enumerate(counts):
        t[j, n:] = float("nan")
        t[j, n + 1:] = float("inf")
    return t


def near(got, want, bound):
    got = wide(got)
    assert got.shape == want.shape and np.isfinite(got).all()
    bad = np.abs(got - want) > bound
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float((np.abs(got - want) / np.maximum(bound, 1e-300)).max()))


# E, C, K, N: around the tiles of 32, 128 and 256 rows and the slabs of 64 and 32, whole numbers of 16 bytes and not, a single row, long buffers
SHAPES = [(3, 5, 64, 64), (1, 1, 8, 8), (2, 1, 1, 1), (4, 33, 72, 40), (3, 130, 200, 136), (5, 64, 128, 256), (2, 300, 256, 264), (3, 17, 33, 35),
          (2, 129, 63, 127), (3, 257, 65, 250), (8, 16, 320, 96), (2, 520, 192, 520), (130, 3, 24, 16), (3, 40, 2056, 24), (2, 31, 100, 500)]


@pytest.mark.parametrize("kind", ["some", "full", "empty"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("E,C,K,N", SHAPES)
def test_products_and_their_gradients(ms, E, C, K, N, dtype, kind):
    print(f"products E={E} C={C} K={K} N={N} {dtype} {kind}", flush=True)
    rng = np.random.default_rng(E * C + K * N)
    counts = counts_of(kind, E, C, rng)
    off, off_h = offsets_of(counts)
    x, xr = normal(rng, (E, C, K), dtype)
    dy, dyr = normal(rng, (E, C, N), dtype)
    spoil(x, counts), spoil(dy, counts)
    for transposed in (False, True):
        w, wr = normal(rng, (E, N, K) if transposed else (E, K, N), dtype, K ** -0.5)
        y, size = ox.expert_matmul(xr, wr, off_h, transposed)
        near(ms.expert_matmul(x, w, off, transposed=transposed), y, HALF[dtype] * np.abs(y) + (K + 1) * STEP32 * size)
        # the gradient of x: the same weights the other way round
        dx, size = ox.expert_matmul(dyr, wr, off_h, not transposed)
        near(ms.expert_matmul(dy, w, off, transposed=not transposed), dx, HALF[dtype] * np.abs(dx) + (N + 1) * STEP32 * size)
    dw, size = ox.expert_matmul_wgrad(xr, dyr, off_h)
    sums = (counts[:, None, None] + 1) * STEP32 * size
    near(ms.expert_matmul_wgrad(x, dy, off), dw, HALF["fp32"] * np.abs(dw) + sums)
    near(ms.expert_matmul_wgrad(dy, x, off), dw.transpose(0, 2, 1), HALF["fp32"] * np.abs(dw.transpose(0, 2, 1)) + sums.transpose(0, 2, 1))
    if dtype == "bf16":
        got = ms.expert_matmul_wgrad(x, dy, off, dtype=torch.bfloat16)
        assert got.dtype == torch.bfloat16
        near(got, dw, HALF["bf16"] * np.abs(dw) + sums)


def swiglu_bound(xr, wr, off_h, transposed, K, N, dtype):
    """The gated unit from sums that are off by eg and eu, a quotient of four fp32 steps, and the rounding of the result.  silu's slope is within 1.1."""
    gu, size = ox.expert_matmul(xr, wr, off_h, transposed)
    sums = (K + 1) * STEP32 * size
    h, silu = ox.swiglu(gu), np.abs(gu[..., :N] * ox.sigmoid(gu[..., :N]))
    eg, eu, u = sums[..., :N], sums[..., N:], np.abs(gu[..., N:])
    return gu, sums, h, HALF[dtype] * np.abs(h) + 1.1 * eg * (u + eu) + silu * eu + 8 * STEP32 * np.abs(h)


@pytest.mark.parametrize("kind", ["some", "full"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("E,C,K,N", SHAPES)
def test_gated_unit_and_its_gradient(ms, E, C, K, N, dtype, kind):
    print(f"swiglu E={E} C={C} K={K} N={N} {dtype} {kind}", flush=True)
    rng = np.random.default_rng(E + C + K + N)
    counts = counts_of(kind, E, C, rng)
    off, off_h = offsets_of(counts)
    x, xr = normal(rng, (E, C, K), dtype)
    spoil(x, counts)
    for transposed in (False, True):
        w, wr = normal(rng, (E, 2 * N, K) if transposed else (E, K, 2 * N), dtype, 2 * K ** -0.5)
        gu, sums, h, bound = swiglu_bound(xr, wr, off_h, transposed, K, N, dtype)
        r = ms.expert_swiglu(x, w, off, transposed=transposed, want_gate_up=True)
        near(r["gate_up"], gu, HALF[dtype] * np.abs(gu) + sums)
        near(r["h"], h, bound)
        alone = ms.expert_swiglu(x, w, off, transposed=transposed)
        assert alone["gate_up"] is None and torch.equal(alone["h"], r["h"])
    gate_up, gur = normal(rng, (E, C, 2 * N), dtype, 3.0)
    dh, dhr = normal(rng, (E, C, N), dtype)
    spoil(gate_up, counts), spoil(dh, counts)
    d, h = ox.swiglu_backward(gur, dhr, off_h)
    got = ms.expert_swiglu_backward(gate_up, dh, off)
    # seven fp32 operations; in 1 + g (1 - s) the terms are up to |g| and cancel near g = -1.28
    g, u = np.abs(gur[..., :N]), np.abs(gur[..., N:])
    near(got["h"], h, HALF[dtype] * np.abs(h) + 8 * STEP32 * np.abs(h))
    keep = (np.arange(C)[None, :] < counts[:, None])[..., None]
    slack = np.concatenate([8 * STEP32 * np.abs(dhr) * u * (1 + g) * keep, 8 * STEP32 * np.abs(d[..., N:])], axis=-1)
    near(got["dgate_up"], d, HALF[dtype] * np.abs(d) + slack)
    alone = ms.expert_swiglu_backward(gate_up, dh, off, want_h=False)
    assert alone["h"] is None and torch.equal(alone["dgate_up"], got["dgate_up"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gated_unit_far_out(ms, dtype):
    """Gates whose exponentials leave fp32 either way give the unit's limits and no NaN."""
    print(f"swiglu far out {dtype}", flush=True)
    g = torch.tensor([-1e30, -1e4, -200.0, -88.0, -1.25, 0.0, 88.0, 200.0, 1e4, 1e30], device="cuda", dtype=torch_type(dtype))
    n = g.numel()
    gate_up = torch.cat([g, torch.ones_like(g)]).reshape(1, 1, 2 * n).contiguous()
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    r = ms.expert_swiglu_backward(gate_up, torch.ones(1, 1, n, device="cuda", dtype=g.dtype), off)
    gd = wide(g)
    s = ox.sigmoid(gd)
    assert np.allclose(wide(r["h"])[0, 0], gd * s, rtol=2 * HALF[dtype] + 1e-6, atol=1e-36)
    assert np.allclose(wide(r["dgate_up"])[0, 0, :n], s * (1 + gd * ox.sigmoid(-gd)), rtol=2 * HALF[dtype] + 1e-6, atol=1e-30)
    # the products' own epilogue: one input column carries the gates, another the ups
    x = torch.ones(1, 1, 8, device="cuda", dtype=g.dtype)
    w = torch.zeros(1, 8, 2 * n, device="cuda", dtype=g.dtype)
    w[0, 0, :n], w[0, 1, n:] = g, 1.0
    assert np.allclose(wide(ms.expert_swiglu(x, w, off)["h"])[0, 0], gd * s, rtol=2 * HALF[dtype] + 1e-6, atol=1e-36)


def dispatch_case(rng, T, E, k, C, ragged=True):
    """Distinct experts per token, places in token order, what does not fit and a few more left empty."""
    assign = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    if ragged:
        assign[rng.random((T, k)) < 0.1] = -1
    pos, fill = np.zeros((T, k), dtype=np.int32), np.zeros(E, dtype=np.int64)
    for i in range(T):
        for s in range(k):
            if assign[i, s] >= 0 and fill[assign[i, s]] >= C:
                assign[i, s] = -1
            if assign[i, s] >= 0:
                pos[i, s] = fill[assign[i, s]]
                fill[assign[i, s]] += 1
    return assign, pos, fill


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d,E,k,C", [(1, 8, 1, 1, 1), (1, 2048, 8, 2, 1), (37, 64, 8, 2, 12), (300, 520, 16, 4, 80), (65, 33, 5, 5, 40), (200, 100, 70, 64, 300),
                                       (1000, 136, 24, 3, 130), (9, 4104, 4, 3, 9), (260, 1, 3, 2, 200), (130, 2056, 20, 6, 64)])
def test_combine_backward(ms, T, d, E, k, C, dtype):
    print(f"combine backward T={T} d={d} E={E} k={k} C={C} {dtype}", flush=True)
    rng = np.random.default_rng(T + d + E)
    assign, pos, fill = dispatch_case(rng, T, E, k, C)
    off, _ = offsets_of(fill)
    eo, eor = normal(rng, (E, C, d), dtype)
    spoil(eo, fill)
    dy, dyr = normal(rng, (T, d), "fp32")
    gates, gr = normal(rng, (T, k), "fp32")
    dev = lambda a: torch.from_numpy(a).cuda()      # noqa: E731
    out = dict(dexpert_out=torch.full_like(eo, 7.0), dgates=torch.full_like(gates, 7.0))
    got = ms.combine_backward(dy, eo, dev(assign), dev(pos), gates, off, out=out)
    de, dg, size = ox.combine_backward(dyr, eor, assign, pos, gr)
    near(got["dexpert_out"], de, (HALF[dtype] + HALF["fp32"]) * (1 + HALF["fp32"]) * np.abs(de))
    near(got["dgates"], dg, HALF["fp32"] * np.abs(dg) + (d + 1) * STEP32 * size)
    # a place outside the buffer is an empty slot
    if T > 1:
        pos2 = pos.copy()
        i, s = np.argwhere(assign >= 0)[-1]
        pos2[i, s] = C
        again = ms.combine_backward(dy, eo, dev(assign), dev(pos2), gates, off)
        assert again["dgates"][i, s].item() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_buffers_that_begin_anywhere(ms, dtype):
    """Rows of whole 16 bytes in buffers that begin off them, and the other way round."""
    print(f"misaligned {dtype}", flush=True)
    rng = np.random.default_rng(3)
    E, C, K, N = 3, 70, 96, 72
    counts = counts_of("some", E, C, rng)
    off, off_h = offsets_of(counts)

    def moved(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    x, xr = normal(rng, (E, C, K), dtype)
    w, wr = normal(rng, (E, K, N), dtype, 0.1)
    dy, dyr = normal(rng, (E, C, N), dtype)
    plain = ms.expert_matmul(x, w, off)
    want, size = ox.expert_matmul(xr, wr, off_h)
    near(plain, want, HALF[dtype] * np.abs(want) + (K + 1) * STEP32 * size)
    for a in (dict(x=moved(x)), dict(w=moved(w)), dict(out=moved(torch.zeros_like(plain)))):
        got = ms.expert_matmul(**dict(dict(x=x, w=w, expert_offsets=off), **a))
        near(got, want, HALF[dtype] * np.abs(want) + (K + 1) * STEP32 * size)
    want, size = ox.expert_matmul_wgrad(xr, dyr, off_h)
    near(ms.expert_matmul_wgrad(moved(x), moved(dy), off), want, HALF["fp32"] * np.abs(want) + (counts[:, None, None] + 1) * STEP32 * size)
    gate_up = moved(ms.expert_swiglu(x, w, off, want_gate_up=True)["gate_up"])
    dh, _ = normal(rng, (E, C, N // 2), dtype)
    a, b = ms.expert_swiglu_backward(gate_up, moved(dh), off), ms.expert_swiglu_backward(gate_up.clone(), dh, off)
    assert torch.equal(a["dgate_up"], b["dgate_up"]) and torch.equal(a["h"], b["h"])


def test_offsets_that_do_not_fit_the_buffers(ms):
    """More rows than places count as the places, a descending pair as none."""
    print("offsets that do not fit", flush=True)
    rng = np.random.default_rng(4)
    x, xr = normal(rng, (4, 6, 16), "bf16")
    w, wr = normal(rng, (4, 16, 24), "bf16")
    off_h = np.array([0, 50, 40, 43, 43], dtype=np.int32)
    off = torch.from_numpy(off_h).cuda()
    want, size = ox.expert_matmul(xr, wr, off_h)
    assert [int(n) for n in ox.rows_of(off_h, 6)] == [6, 0, 3, 0]
    near(ms.expert_matmul(x, w, off), want, HALF["bf16"] * np.abs(want) + 17 * STEP32 * size)
    dy, dyr = normal(rng, (4, 6, 24), "bf16")
    want, size = ox.expert_matmul_wgrad(xr, dyr, off_h)
    near(ms.expert_matmul_wgrad(x, dy, off), want, HALF["fp32"] * np.abs(want) + 7 * STEP32 * size)


def test_infinities_and_nans_stay_in_their_rows_and_columns(ms):
    print("infinities", flush=True)
    rng = np.random.default_rng(5)
    E, C, K, N = 2, 150, 72, 40
    off, off_h = offsets_of([C, 90])
    x, _ = normal(rng, (E, C, K), "bf16")
    w, _ = normal(rng, (E, K, N), "bf16")
    clean = ms.expert_matmul(x, w, off)
    x2, w2 = x.clone(), w.clone()
    x2[0, 7, 71], x2[1, 33, 0], w2[0, 70, 11] = float("inf"), float("nan"), float("-inf")
    got = ms.expert_matmul(x2, w2, off)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[0, 7, :], hit[1, 33, :], hit[0, :, 11] = True, True, True
    assert torch.equal(got[~hit], clean[~hit])
    assert not torch.isfinite(got[0, 7]).any() and torch.isnan(got[1, 33]).all() and not torch.isfinite(got[0, :, 11]).any()


@pytest.mark.parametrize("E,C,K,N,dtype", [(16, 512, 1024, 1024, "bf16"), (8, 300, 1000, 504, "fp32"), (64, 40, 2048, 512, "bf16"), (4, 2048, 2048, 512, "bf16")])
def test_products_of_layers(ms, E, C, K, N, dtype):
    """Sizes of layers, the oracle in 64 bits on the GPU."""
    print(f"layers E={E} C={C} K={K} N={N} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(C)
    counts = torch.randint(0, C + 1, (E,), generator=gen, device="cuda")
    counts[0] = C
    off = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
    keep = (torch.arange(C, device="cuda")[None, :] < counts[:, None])[..., None]
    draw = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch_type(dtype))       # noqa: E731
    x, dy, w = draw(E, C, K), draw(E, C, N), draw(E, K, N)
    xd, dyd, wd = x.double() * keep, dy.double() * keep, w.double()

    def check(got, a, b, half, terms):
        want, size = a @ b, a.abs() @ b.abs()
        assert bool(((got.double() - want).abs() <= half * want.abs() + (terms + 1) * STEP32 * size).all())

    check(ms.expert_matmul(x, w, off), xd, wd, HALF[dtype], K)
    check(ms.expert_matmul(x, w.transpose(1, 2).contiguous(), off, transposed=True), xd, wd, HALF[dtype], K)
    check(ms.expert_matmul(dy, w, off, transposed=True), dyd, wd.transpose(1, 2).contiguous(), HALF[dtype], N)
    check(ms.expert_matmul_wgrad(x, dy, off), xd.transpose(1, 2).contiguous(), dyd, HALF["fp32"], C)
    r = ms.expert_swiglu(x, w, off, want_gate_up=True)
    check(r["gate_up"], xd, wd, HALF[dtype], K)
    again = ms.expert_swiglu(x, w, off, want_gate_up=True)
    assert torch.equal(r["h"], again["h"]) and torch.equal(r["gate_up"], again["gate_up"])       # the same every time


def layer(ms, x, W, w_in, w_out, k, C, d_out):
    """One layer forward and back by the library alone: the gradients of sum(y * d_out) with the assignment held."""
    T, d = x.shape
    E = W.shape[1]
    r = ms.route_xw(x, W, None, k, C)
    off, assign, pos, gates = r["expert_offsets"], r["assign"], r["token_pos"], r["gates"]
    xin = ms.dispatch_tokens(x, off, r["disp_token"], E, C)
    mid = ms.expert_swiglu(xin, w_in, off, want_gate_up=True)
    out = ms.expert_matmul(mid["h"], w_out, off)
    y = ms.combine(out, assign, pos, gates)
    back = ms.combine_backward(d_out, out, assign, pos, gates, off)
    dout = back["dexpert_out"]
    dw_out = ms.expert_matmul_wgrad(mid["h"], dout, off)
    dh = ms.expert_matmul(dout, w_out, off, transposed=True)
    act = ms.expert_swiglu_backward(mid["gate_up"], dh, off)
    dw_in = ms.expert_matmul_wgrad(xin, act["dgate_up"], off)
    dxin = ms.expert_matmul(act["dgate_up"], w_in, off, transposed=True)
    dx = ms.combine(dxin, assign, pos, torch.ones_like(gates))
    return dict(r=r, y=y, dgates=back["dgates"], dw_out=dw_out, dw_in=dw_in, dx=dx, h=mid["h"], act_h=act["h"])


def test_a_layer_forward_and_back(ms):
    """Routing, rows out, gated unit, product, rows back and the way back through all of them in fp32, against the same in 64 bits and against
    differences of the 64-bit loss.  Everything is fp32: relative errors of sums of up to a few hundred terms, some 1e-5 through five steps."""
    print("layer forward and back", flush=True)
    rng = np.random.default_rng(9)
    T, d, E, k, n = 300, 72, 8, 2, 40
    C = 90
    x, xr = normal(rng, (T, d), "fp32")
    W, _ = normal(rng, (d, E), "fp32", d ** -0.5)
    w_in, wir = normal(rng, (E, d, 2 * n), "fp32", d ** -0.5)
    w_out, wor = normal(rng, (E, n, d), "fp32", n ** -0.5)
    d_out, dor = normal(rng, (T, d), "fp32")
    got = layer(ms, x, W, w_in, w_out, k, C, d_out)
    r = got["r"]
    assign, pos, gates = r["assign"].cpu().numpy(), r["token_pos"].cpu().numpy(), wide(r["gates"])
    off, tok = r["expert_offsets"].cpu().numpy(), r["disp_token"].cpu().numpy()

    def forward(x_, g_, wi_, wo_):
        xin = oracle.dispatch_tokens(x_, off, tok, E, C)
        gu, _ = ox.expert_matmul(xin, wi_, off)
        h = ox.swiglu(gu)
        out, _ = ox.expert_matmul(h, wo_, off)
        return xin, gu, h, out, oracle.combine(out, assign, pos, g_)

    xin, gu, h, out, y = forward(xr, gates, wir, wor)
    de, dg, _ = ox.combine_backward(dor, out, assign, pos, gates)
    dwo, _ = ox.expert_matmul_wgrad(h, de, off)
    dgu, _ = ox.swiglu_backward(gu, ox.expert_matmul(de, wor, off, True)[0], off)
    dwi, _ = ox.expert_matmul_wgrad(xin, dgu, off)
    dx = oracle.combine(ox.expert_matmul(dgu, wir, off, True)[0], assign, pos, np.ones_like(gates))

    def close(a, b):
        a = wide(a)
        assert np.abs(a - b).max() <= 2e-5 * np.abs(b).max(), np.abs(a - b).max() / np.abs(b).max()

    for a, b in ((got["y"], y), (got["dgates"], dg), (got["dw_out"], dwo), (got["dw_in"], dwi), (got["dx"], dx), (got["h"], h), (got["act_h"], h)):
        close(a, b)
    loss = lambda *a: (forward(*a)[-1] * dor).sum()       # noqa: E731
    args = [xr, gates, wir, wor]
    for i, grad in enumerate((got["dx"], got["dgates"], got["dw_in"], got["dw_out"])):
        v = rng.normal(size=args[i].shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * v, args[i] - 1e-5 * v
        want = (loss(*up) - loss(*down)) / 2e-5
        assert abs((wide(grad) * v).sum() - want) <= 1e-4 * max(1.0, abs(want)), i


def expert_steps(ms, s):
    a = ms.expert_swiglu(s["x"], s["w"], s["off"], want_gate_up=True)
    b = ms.expert_matmul(a["h"], s["w2"], s["off"])
    back = ms.combine_backward(s["dy"], b, s["assign"], s["pos"], s["gates"], s["off"])
    dh = ms.expert_matmul(back["dexpert_out"], s["w2"], s["off"], transposed=True)
    c = ms.expert_swiglu_backward(a["gate_up"], dh, s["off"])
    q, scales = ms.mxfp4_quantise(a["h"])
    return [a["h"], a["gate_up"], b, back["dexpert_out"], back["dgates"], c["dgate_up"], c["h"], ms.expert_matmul_wgrad(s["x"], c["dgate_up"], s["off"]), q, scales,
            ms.expert_matmul_mxfp4(q, scales, s["wq"], s["ws"], s["off"]), ms.mxfp4_dequantise(q, scales)]


def steps_state(ms, seed, C):
    rng = np.random.default_rng(seed)
    T, E, k, d, n = 200, 8, 2, 128, 96
    assign, pos, fill = dispatch_case(rng, T, E, k, C)
    off, _ = offsets_of(fill)
    s = dict(off=off, assign=torch.from_numpy(assign).cuda(), pos=torch.from_numpy(pos).cuda())
    for name, shape, dtype in (("x", (E, C, d), "bf16"), ("w", (E, d, 2 * n), "bf16"), ("w2", (E, n, d), "bf16"), ("dy", (T, d), "fp32"), ("gates", (T, k), "fp32")):
        s[name] = normal(rng, shape, dtype, 0.2)[0]
    s["wq"], s["ws"] = ms.mxfp4_quantise(s["w2"].transpose(1, 2).contiguous())
    return s


def test_captured_and_replayed(ms):
    """A captured chain of the calls, replayed between eager work of other sizes and with new inputs in its buffers, gives the eager results."""
    print("captured", flush=True)
    s, other = steps_state(ms, 1, 60), steps_state(ms, 2, 300)
    expert_steps(ms, s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = expert_steps(ms, s)
    for seed in range(3):
        fresh = steps_state(ms, 10 + seed, 60)
        for name in s:
            s[name].copy_(fresh[name])
        g.replay()
        between = expert_steps(ms, other)
        torch.cuda.synchronize()
        for a, b in zip(out, expert_steps(ms, s)):
            assert torch.equal(a, b)
        for a, b in zip(between, expert_steps(ms, other)):
            assert torch.equal(a, b)


def test_calls_on_two_streams_at_once(ms):
    print("two streams", flush=True)
    s, t = steps_state(ms, 3, 60), steps_state(ms, 4, 130)
    want = [expert_steps(ms, s), expert_steps(ms, t)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for i, (stream, state) in enumerate(zip(streams, (s, t))):
        with torch.cuda.stream(stream):
            got[i] = [expert_steps(ms, state) for _ in range(4)]
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            for a, b in zip(run, want[i]):
                assert torch.equal(a, b)


def test_buffers_past_32_bits(ms):
    """Rows of experts whose buffers lie beyond 4 GiB and beyond 2^31 elements."""
    print("past 32 bits", flush=True)
    E, C, K, N = 3, 1 << 20, 1032, 8
    x = torch.zeros((E, C, K), dtype=torch.bfloat16, device="cuda")
    w = torch.randn((E, K, N), device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, C, 2 * C, 3 * C], dtype=torch.int32, device="cuda")
    rows = [0, 1, C // 2 + 5, C - 1]
    for j in range(E):
        x[j, rows] = torch.randn((4, K), device="cuda").to(torch.bfloat16)
    y = ms.expert_matmul(x, w, off)
    for j in range(E):
        want = x[j, rows].double() @ w[j].double()
        size = x[j, rows].double().abs() @ w[j].double().abs()
        assert bool(((y[j, rows].double() - want).abs() <= HALF["bf16"] * want.abs() + (K + 1) * STEP32 * size).all())
        assert not y[j, 2:1000].any() and not y[j, C - 1000:C - 1].any()
    dx = ms.expert_matmul(y, w, off, transposed=True)
    for j in range(E):
        want = y[j, rows].double() @ w[j].double().T
        size = y[j, rows].double().abs() @ w[j].double().abs().T
        assert bool(((dx[j, rows].double() - want).abs() <= HALF["bf16"] * want.abs() + 9 * STEP32 * size).all())
