"""The experts' products, the gated unit, their gradients and microscaled four-bit rows in 64 bits (numpy), from their definitions."""
import numpy as np

MX_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rows_of(expert_offsets, C):
    off = np.asarray(expert_offsets, dtype=np.int64)
    return np.clip(off[1:] - off[:-1], 0, C)


def expert_matmul(x, W, expert_offsets, transposed=False):
    """(y, sum of |x||W| per entry): every expert's rows times its weights, zero rows behind them."""
    x, W = np.asarray(x, dtype=np.float64), np.asarray(W, dtype=np.float64)
    W = W.transpose(0, 2, 1) if transposed else W
    E, C, _ = x.shape
    y, size = np.zeros((E, C, W.shape[2])), np.zeros((E, C, W.shape[2]))
    for j, n in enumerate(rows_of(expert_offsets, C)):
        y[j, :n] = x[j, :n] @ W[j]
        size[j, :n] = np.abs(x[j, :n]) @ np.abs(W[j])
    return y, size


def expert_matmul_wgrad(x, dy, expert_offsets):
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    E, C, K = x.shape
    dw, size = np.zeros((E, K, dy.shape[2])), np.zeros((E, K, dy.shape[2]))
    for j, n in enumerate(rows_of(expert_offsets, C)):
        dw[j] = x[j, :n].T @ dy[j, :n]
        size[j] = np.abs(x[j, :n]).T @ np.abs(dy[j, :n])
    return dw, size


def sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0, e) / (1.0 + e)


def swiglu(gate_up):
    n = gate_up.shape[-1] // 2
    g, u = gate_up[..., :n], gate_up[..., n:]
    return u * g * sigmoid(g)


def swiglu_backward(gate_up, dh, expert_offsets):
    gate_up, dh = np.asarray(gate_up, dtype=np.float64), np.asarray(dh, dtype=np.float64)
    E, C, n = dh.shape
    out, h = np.zeros((E, C, 2 * n)), np.zeros((E, C, n))
    for j, r in enumerate(rows_of(expert_offsets, C)):
        g, u, d = gate_up[j, :r, :n], gate_up[j, :r, n:], dh[j, :r]
        s = sigmoid(g)
        out[j, :r, :n] = d * u * s * (1.0 + g * sigmoid(-g))
        out[j, :r, n:] = d * g * s
        h[j, :r] = u * g * s
    return out, h


def combine_backward(dy, expert_out, assign, token_pos, gates):
    """(dexpert_out, dgates, sum of |dy||expert_out| per gate)."""
    dy, eo = np.asarray(dy, dtype=np.float64), np.asarray(expert_out, dtype=np.float64)
    E, C, _ = eo.shape
    dexpert_out, dgates, size = np.zeros_like(eo), np.zeros(assign.shape), np.zeros(assign.shape)
    for i in range(assign.shape[0]):
        for s in range(assign.shape[1]):
            e, p = assign[i, s], token_pos[i, s]
            if e < 0 or e >= E or p < 0 or p >= C:
                continue
            dexpert_out[e, p] = float(gates[i, s]) * dy[i]
            dgates[i, s] = dy[i] @ eo[e, p]
            size[i, s] = np.abs(dy[i]) @ np.abs(eo[e, p])
    return dexpert_out, dgates, size


def mxfp4_quantise(x):
    """(codes uint8 [..., d], scale bytes uint8 [..., d/32]): each value's nearest number of the grid, found by trying all of them."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    codes, scales = np.zeros(blocks.shape, dtype=np.uint8), np.zeros(blocks.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(*scales.shape):
        b = blocks[at]
        if not np.isfinite(b).all():
            scales[at] = 255
            continue
        top = np.abs(b).max()
        exponent = -127 if top == 0 else max(-127, int(np.frexp(top)[1]) - 1 - 2)
        scales[at] = exponent + 127
        v = np.ldexp(np.abs(b), -exponent)
        far = np.abs(v[:, None] - MX_GRID)
        best = far.min(axis=1, keepdims=True)
        for i in range(32):
            near = np.nonzero(far[i] == best[i])[0]
            codes[at][i] = (near[0] if len(near) == 1 else near[near % 2 == 0][0]) + (8 if np.signbit(b[i]) else 0)
    return codes.reshape(x.shape), scales


def mxfp4_values(codes, scales):
    v = np.where(codes & 8, -1.0, 1.0) * MX_GRID[codes & 7]
    with np.errstate(invalid="ignore"):
        scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(*scales.shape, 32) * scale[..., None]).reshape(codes.shape)


def mxfp4_pack(codes):
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def mxfp4_unpack(q):
    return np.stack([q & 15, q >> 4], axis=-1).reshape(*q.shape[:-1], -1)
