"""The operators of a quantized state-space block in 64 bits, from their
definitions (numpy), with bounds on the rounding of an fp32 evaluation.  U32 is
half a step of fp32 relative to the value, HALF the same of the three types."""
import numpy as np
import torch

U32 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# half the smallest step of a type (results near 0)
TINY = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
TYPES = (torch.float32, torch.float16, torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


def half_up(v):
    r = np.floor(v)
    return r + ((v - r) >= 0.5)


def quantize8(Y):
    """Rows of Y (fp32 values): codes 0..255, zero points, recovery factors fp32."""
    Y = np.asarray(Y, np.float64)
    lo, hi = Y.min(1), Y.max(1)
    R, top = hi - lo, np.maximum(np.abs(lo), np.abs(hi))
    narrow = (R == 0) | (255 * top > 16777216.0 * R)
    lo, hi = np.where(narrow, np.minimum(lo, 0), lo), np.where(narrow, np.maximum(hi, 0), hi)
    R = hi - lo
    Q = np.where(R == 0, 1.0, 255 / np.where(R == 0, 1.0, R))
    z = np.where(R == 0, 0, half_up(Q * lo))
    codes = np.clip(half_up(Q[:, None] * Y) - z[:, None], 0, 255)
    return codes.astype(np.uint8), z.astype(np.int32), np.where(R == 0, 1.0, R / 255).astype(np.float32)


def quantize4(W, group):
    """Codes 0..15 [rows][cols], zero points and recovery factors [rows][groups]."""
    W = np.asarray(W, np.float64)
    rows, cols = W.shape
    n = -(-cols // group)
    V = np.zeros((rows, n * group))
    V[:, :cols] = W
    V = V.reshape(rows, n, group)
    lo, hi = np.minimum(V.min(2), 0), np.maximum(V.max(2), 0)
    R = hi - lo
    Q = np.where(R == 0, 1.0, 15 / np.where(R == 0, 1.0, R))
    z = np.where(R == 0, 0, half_up(Q * lo))
    codes = np.clip(half_up(Q[..., None] * V) - z[..., None], 0, 15).reshape(rows, -1)[:, :cols]
    return codes.astype(np.uint8), z.astype(np.int8), np.where(R == 0, 1.0, R / 15).astype(np.float32)


def matmul4(codes, zero, inv_q, group, xcodes, xzero, xinv_q):
    """(Y, bound): the product in 64 bits, and how far an fp32 sum over groups with
    one rounding of each T_g may be from it, in any order of the groups."""
    cols = codes.shape[1]
    W2 = codes.astype(np.float64) + np.repeat(zero.astype(np.float64), group, 1)[:, :cols]
    X2 = xcodes.astype(np.float64) + xzero.astype(np.float64)[:, None]
    n = zero.shape[1]
    Y = np.zeros((X2.shape[0], W2.shape[0]))
    mag = np.zeros_like(Y)
    for g in range(n):
        k = slice(g * group, min((g + 1) * group, cols))
        # parts of a group may be summed on their own: their magnitudes count
        t = np.zeros_like(Y)
        for k0 in range(k.start, k.stop, 32):
            kk = slice(k0, min(k0 + 32, k.stop))
            part = X2[:, kk] @ W2[:, kk].T
            t += part
            mag += np.abs(part) * inv_q[:, g].astype(np.float64)
        Y += t * inv_q[:, g].astype(np.float64)
    qx = xinv_q.astype(np.float64)[:, None]
    # a part's rounding, its product's, up to 4 n additions, and qx's
    return Y * qx, (4 * n + 4) * U32 * mag * qx


def rms_norm_backward(dy, v, rstd, w, dsum, terms):
    """(dx, bound, dw, bound) with sums of `terms` sequential fp32 additions at most."""
    n = dy.shape[1]
    g = dy * w
    r = rstd[:, None]
    s, sa = (g * v).sum(1, keepdims=True), np.abs(g * v).sum(1, keepdims=True)
    dx = r * g - v * r ** 3 / n * s + (0 if dsum is None else dsum)
    bx = U32 * (4 * np.abs(r * g) + np.abs(v) * r ** 3 / n * ((terms + 8) * sa + 8 * np.abs(s))
                + 2 * np.abs(dx) + (0 if dsum is None else np.abs(dsum)))
    dw = (dy * (v * r)).sum(0)
    bw = U32 * (dy.shape[0] + 4) * np.abs(dy * (v * r)).sum(0)
    return dx, bx, dw, bw


def clamp_lengths(lengths, T, B):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)


def conv(x, w, b, silu, lengths, state):
    """(y, bound, state): rows past a sequence's length are 0."""
    T, B, D = x.shape
    W = w.shape[0]
    n = clamp_lengths(lengths, T, B)
    xp = np.concatenate([state.transpose(1, 0, 2), x])
    s, mag = np.zeros((T, B, D)) + b, np.zeros((T, B, D)) + np.abs(b)
    for j in range(W):
        s, mag = s + w[j] * xp[j:j + T], mag + np.abs(w[j] * xp[j:j + T])
    bs = U32 * (W + 1) * mag
    if silu:
        # silu's slope is below 1.1; e^-x, the sum and the division round 6 times
        y = s / (1 + np.exp(-s))
        bound = 1.1 * bs + 8 * U32 * np.abs(y) + U32 * np.abs(s) * np.abs(y)
    else:
        y, bound = s, bs
    out = np.stack([xp[n[i]:n[i] + W - 1, i] for i in range(B)]) if B else state.copy()
    on = (np.arange(T)[:, None] < n)[..., None]
    return np.where(on, y, 0), np.where(on, bound, 0), out


def scan(u, delta, A, Bm, Cm, D, z, bias, softplus, lengths, state):
    """(y, bound, state, bound).  The bound follows an fp32 evaluation: e^x off by
    (|x| + 4) half steps, softplus by 8, and sums of up to 256 steps' d in fp32
    where the scan is split over time (256 half steps of their argument)."""
    T, B, C = u.shape
    n = clamp_lengths(lengths, T, B)
    h, E = state.copy(), np.zeros_like(state)
    y, by = np.zeros((T, B, C)), np.zeros((T, B, C))
    for t in range(T):
        on = (t < n)[:, None, None]
        d0 = delta[t] + bias
        d = np.logaddexp(d0, 0) if softplus else d0
        # d's error: its sum's rounding times the slope (at most 1), and 8 of its own
        bd = U32 * (np.abs(d0) + 8 * np.abs(d)) if softplus else U32 * np.abs(d0)
        dA = d[:, None, :] * A
        a = np.exp(dA)
        ea = U32 * (260 * np.abs(dA) + 8) + bd[:, None, :] * np.abs(A)
        x = (d * u[t])[:, None, :] * Bm[t][:, :, None]
        ex = (bd * np.abs(u[t]))[:, None, :] * np.abs(Bm[t][:, :, None]) + 4 * U32 * np.abs(x)
        nh = a * h + x
        nE = a * (E * (1 + 2 * ea) + 1.1 * ea * np.abs(h)) + ex + 4 * U32 * (np.abs(nh) + a * np.abs(h))
        h, E = np.where(on, nh, h), np.where(on, nE, E)
        terms = Cm[t][:, :, None] * h
        s = terms.sum(1) + D * u[t]
        bs = (np.abs(Cm[t][:, :, None]) * E).sum(1) \
            + U32 * (A.shape[0] + 4) * (np.abs(terms).sum(1) + np.abs(D * u[t]))
        if z is not None:
            zz = z[t]
            g = zz / (1 + np.exp(-zz))
            s, bs = s * g, bs * np.abs(g) + U32 * (10 + np.abs(zz)) * np.abs(s * g)
        y[t], by[t] = np.where(on[:, 0], s, 0), np.where(on[:, 0], bs, 0)
    return y, by, h, E


def close(got, want, bound, dtype, what):
    """got (a tensor of dtype) within the fp32 evaluation's bound and its own rounding."""
    got = f64(got)
    tol = bound * (1 + 2 * HALF[dtype]) + HALF[dtype] * np.abs(want) * (1 if dtype != torch.float32 else 2) \
        + TINY[dtype] * 2
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                           got[bad][:3], want[bad][:3], tol[bad][:3])
