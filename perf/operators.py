"""The operators of a quantized state-space block, as timed cases: the
root-mean-square norm with the residual's addition (float output or 8-bit
codes, and its backward pass), products with 4-bit weights and group scales,
and the selective scan with its short causal convolution, for prompts and for
single tokens.

`run` computes a case in its plain form (elementary torch operations) or, with
`own` set, through the public entry points of paper_1607_04683_amd.qlstm.
Inputs are synthetic: activations N(0, 1), weights N(0, 0.02), steps
softplus(delta + bias) around 0.001 to 0.1, decay rates -1 to -16.

Sequences are time-major, [T][B][channels], as everywhere in this repository.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


# ------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of a stream: residual added, normed and quantized for the
        # product that follows; the smallest call, where latency counts
        dict(name="norm_token_1x2048", kind="norm", m=1, cols=2048, type="f32", residual=True,
             out="codes"),
        # a long prompt in bfloat16, the same call
        dict(name="norm_prompt_4096x4096_bf16", kind="norm", m=4096, cols=4096, type="bf16",
             residual=True, out="codes"),
        # the frames of the benchmark's batch (64 utterances of 30 s) at the
        # width of its layers, float output for a float layer, as training keeps it
        dict(name="norm_frames_64000x500", kind="norm", m=64000, cols=500, type="f32",
             residual=False, out="y"),
        # the backward pass of the training step's batch (64 x 200 frames)
        dict(name="norm_grad_12800x500", kind="grad", m=12800, cols=500, type="f32",
             residual=True),
        # the backward pass of a long prompt in bfloat16
        dict(name="norm_grad_4096x4096_bf16", kind="grad", m=4096, cols=4096, type="bf16",
             residual=True),
        # one token through a projection, its activations in codes already (from the norm)
        dict(name="q4_token_1x2048x8192_g128", kind="q4", m=1, cols=2048, rows=8192, group=128,
             type="f32", x="codes", bias=False),
        # a few streams through one layer's input product, odd sizes, fp32 rows
        # quantized on the fly
        dict(name="q4_few_6x500x2000_g32", kind="q4", m=6, cols=500, rows=2000, group=32,
             type="f32", x="rows", bias=True),
        # a decoding batch through a wide output layer
        dict(name="q4_batch_64x4096x16384_g64", kind="q4", m=64, cols=4096, rows=16384, group=64,
             type="bf16", x="rows", bias=False),
        # one token of one stream, state carried
        dict(name="ssm_token_b1_d1024", kind="ssm", T=1, B=1, D=1024, N=16, W=4, type="f32",
             ragged=False),
        # one token of each of 64 streams
        dict(name="ssm_token_b64_d4096_bf16", kind="ssm", T=1, B=64, D=4096, N=16, W=4,
             type="bf16", ragged=False),
        # one long prompt
        dict(name="ssm_prompt_b1_t4096_d2048_bf16", kind="ssm", T=4096, B=1, D=2048, N=16, W=4,
             type="bf16", ragged=False),
        # a padded batch of prompts of different lengths, an odd width
        dict(name="ssm_batch_b12_t1000_d1000", kind="ssm", T=1000, B=12, D=1000, N=16, W=4,
             type="f32", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "grad", "q4", "q4", "ssm", "ssm"])
    type_ = rng.choice(["f32", "f16", "bf16"])
    if kind in ("norm", "grad"):
        cols = _log(rng, 64, 8192)
        m = _log(rng, 1, min(64000, (1 << 24) // cols))
        c = dict(kind=kind, m=m, cols=cols, type=type_, residual=rng.random() < 0.6)
        return c if kind == "grad" else dict(c, out=rng.choice(["codes", "codes", "y"]))
    if kind == "q4":
        return dict(kind=kind, m=_log(rng, 1, 64), cols=_log(rng, 64, 4096),
                    rows=_log(rng, 64, 16384), group=rng.choice([32, 64, 128]), type=type_,
                    x=rng.choice(["codes", "rows"]), bias=rng.random() < 0.5)
    N, D = rng.choice([8, 16, 16, rng.randint(1, 32)]), _log(rng, 64, 4096)
    W = rng.choice([4, 4, 2, 3])
    if rng.random() < 0.4:
        return dict(kind=kind, T=1, B=_log(rng, 1, 64), D=D, N=N, W=W, type=type_, ragged=False)
    B = _log(rng, 1, 16)
    T = _log(rng, 2, max(2, min(4096, (1 << 27) // (B * D * N))))
    return dict(kind=kind, T=T, B=B, D=D, N=N, W=W, type=type_, ragged=rng.random() < 0.5)


# --------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _half_up(v):
    """round() of the quantizer: half up, decided exactly (fp64)."""
    r = torch.floor(v)
    return r + ((v - r) >= 0.5)


def _codes8(V):
    """The per-vector 8-bit quantizer in fp64: rows of V -> (codes 0..255, zero
    points, recovery factors)."""
    V = V.double()
    lo, hi = V.amin(1, keepdim=True), V.amax(1, keepdim=True)
    R, top = hi - lo, torch.maximum(lo.abs(), hi.abs())
    narrow = (R == 0) | (255 * top > 16777216 * R)
    lo, hi = torch.where(narrow, lo.clamp(max=0), lo), torch.where(narrow, hi.clamp(min=0), hi)
    R = hi - lo
    none = R == 0
    Q = torch.where(none, 1.0, 255 / torch.where(none, 1.0, R))
    z = torch.where(none, 0.0, _half_up(Q * lo))
    return ((_half_up(Q * V) - z).clamp(0, 255), z, torch.where(none, 1.0, R / 255).float())


def _codes4(W, group):
    """The 4-bit group quantizer: W [rows][cols] -> codes 0..15 [rows][ld], zero
    points and recovery factors [rows][ld / group]; ld a multiple of 128, what is
    padded recovers to 0.  The range of a group holds 0."""
    rows, cols = W.shape
    ld = (cols + 127) // 128 * 128
    V = torch.zeros(rows, ld, dtype=torch.float64, device=DEV)
    V[:, :cols] = W
    V = V.reshape(rows, ld // group, group)
    lo, hi = V.amin(2, keepdim=True).clamp(max=0), V.amax(2, keepdim=True).clamp(min=0)
    R = hi - lo
    none = R == 0
    Q = torch.where(none, 1.0, 15 / torch.where(none, 1.0, R))
    z = torch.where(none, 0.0, _half_up(Q * lo))
    codes = (_half_up(Q * V) - z).clamp(0, 15)
    return (codes.reshape(rows, ld).to(torch.uint8), z[:, :, 0].to(torch.int8),
            torch.where(none, 1.0, R / 15).float()[:, :, 0])


def _pack4(codes):
    """Codes 0..15 [rows][ld] -> bytes [rows][ld / 2] of the 4-bit layout: in every
    128 columns word 4 q + p holds columns 32 p + 8 q .. + 7, byte j of a word
    columns j (low half) and j + 4 (high half), each half V' - 8 in two's complement."""
    rows, ld = codes.shape
    c = (codes ^ 8).reshape(rows, ld // 128, 4, 4, 2, 4).permute(0, 1, 3, 2, 4, 5)
    return (c[..., 0, :] | (c[..., 1, :] << 4)).reshape(rows, ld // 2).contiguous()


def _unpack4(packed):
    rows, n = packed.shape
    w = packed.reshape(rows, n // 64, 4, 4, 1, 4)
    c = torch.cat([w & 15, w >> 4], 4) ^ 8
    return c.permute(0, 1, 3, 2, 4, 5).reshape(rows, 2 * n)


def _by_group(v, rows):
    """[rows][groups] -> the layout [groups][rows up to a multiple of 16]."""
    out = torch.zeros(v.shape[1], (rows + 15) // 16 * 16, dtype=v.dtype, device=DEV)
    out[:, :rows] = v.T
    return out


def _signed8(codes):
    """Codes 0..255 [rows][cols] -> int8 [rows][ld] of the 8-bit layout."""
    rows, cols = codes.shape
    out = torch.zeros(rows, (cols + 63) // 64 * 64, dtype=torch.int8, device=DEV)
    out[:, :cols] = (codes.to(torch.int32) - 128).to(torch.int8)
    return out


def _draw_inputs(case, seed):
    g, c, k = _gen(seed), case, case["kind"]
    dt = TYPES[c["type"]]
    z = lambda *s: torch.randn(*s, generator=g, device=DEV)
    u = lambda *s: torch.rand(*s, generator=g, device=DEV)
    if k in ("norm", "grad"):
        m, n = c["m"], c["cols"]
        d = dict(x=z(m, n).to(dt), weight=1 + 0.1 * z(n),
                 residual=(2 * z(m, n)).to(dt) if c["residual"] else None)
        if k == "grad":
            d["dy"] = z(m, n).to(dt)
            d["rstd"] = (1 / torch.sqrt(d["x"].double().square().mean(1) + EPS)).float()
        return d
    if k == "q4":
        return dict(W=z(c["rows"], c["cols"]) * 0.02, X=z(c["m"], c["cols"]).to(dt),
                    bias=0.1 * z(c["rows"]) if c["bias"] else None)
    T, B, D, N, W = c["T"], c["B"], c["D"], c["N"], c["W"]
    step = torch.exp(math.log(0.001) + u(D) * math.log(100.0))
    d = dict(x=z(T, B, D).to(dt), w=z(W, D) * 0.4, b=z(D) * 0.1, conv_state=z(B, W - 1, D),
             u=z(T, B, D).to(dt), delta=(0.5 * z(T, B, D)).to(dt),
             delta_bias=torch.log(torch.expm1(step)), A=-torch.exp(u(N, D) * math.log(16.0)),
             Bm=z(T, B, N).to(dt), Cm=z(T, B, N).to(dt), Dskip=z(D), z=z(T, B, D).to(dt),
             state=0.1 * z(B, N, D), lengths=None)
    if c["ragged"]:  # one full length, the others anywhere down to none
        n = torch.floor(u(B) * (T + 1)).to(torch.int32)
        n[0] = T
        d["lengths"] = n
    return d


def prepare(case, seed):
    d, c, k = _draw_inputs(case, seed), case, case["kind"]
    dt = TYPES[c["type"]]
    s = dict(d, case=case)
    if k == "q4":
        codes, zero, inv_q = _codes4(d["W"], c["group"])
        s.update(packed=_pack4(codes), zero=_by_group(zero, c["rows"]),
                 inv_q=_by_group(inv_q, c["rows"]))
        del s["W"]
        if c["x"] == "codes":
            v, z, iq = _codes8(s.pop("X").float())
            s.update(xcodes=_signed8(v), xzero=z[:, 0].to(torch.int32),
                     xinv_q=iq[:, 0].contiguous(), xsums=v.sum(1).to(torch.int32))
    if k == "ssm":  # the program's buffers: what lies behind a sequence's end stays as it is
        s.update(conv_out=torch.zeros_like(d["x"]), y=torch.zeros_like(d["u"]),
                 conv_state_out=torch.zeros_like(d["conv_state"]),
                 state_out=torch.zeros_like(d["state"]), ws=None)
    return s


# ------------------------------------------------------------ the plain forms
def _sum_type(x, residual):
    return x if residual is None else (x.float() + residual.float()).to(x.dtype)


def _plain_norm(s):
    c = s["case"]
    v = _sum_type(s["x"], s["residual"])
    ms = v.double().square().sum(1, keepdim=True) / c["cols"]
    rstd = torch.reciprocal(torch.sqrt(ms + EPS)).float()
    y = (v.float() * rstd) * s["weight"]
    out = dict(sum=v) if s["residual"] is not None else {}
    if c["out"] == "y":
        return dict(out, y=y.to(v.dtype), rstd=rstd[:, 0])
    codes, zero, inv_q = _codes8(y)
    return dict(out, recovered=(codes + zero).float() * inv_q)


def _plain_grad(s):
    v, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    g = dy * s["weight"]
    c1 = (g * v).sum(1, keepdim=True) * (rstd * rstd * rstd / s["case"]["cols"])
    dx = g * rstd - v * c1
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dict(dx=dx.to(s["x"].dtype), dweight=(dy * (v * rstd)).sum(0))


def _plain_q4(s):
    c = s["case"]
    rows, cols, group = c["rows"], c["cols"], c["group"]
    spread = lambda v: v[:, :rows].T.float().repeat_interleave(group, 1)
    W = ((_unpack4(s["packed"]).float() + spread(s["zero"])) * spread(s["inv_q"]))[:, :cols]
    if c["x"] == "codes":
        X = (s["xcodes"][:, :cols].float() + (s["xzero"][:, None] + 128).float()) * s["xinv_q"][:, None]
    else:
        codes, zero, inv_q = _codes8(s["X"].float())
        X = (codes + zero).float() * inv_q
    Y = X @ W.T
    if s["bias"] is not None:
        Y = Y + s["bias"]
    return Y.to(TYPES[c["type"]])


def _valid(c, lengths):
    """[T][B][1]: the steps within their sequence."""
    t = torch.arange(c["T"], device=DEV)[:, None]
    n = torch.full((c["B"],), c["T"], device=DEV) if lengths is None else lengths
    return (t < n).unsqueeze(2), n.long()


def _silu(v):
    return v / (1 + torch.exp(-v))


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _plain_conv(s, valid, n):
    c = s["case"]
    T, W = c["T"], c["W"]
    xp = torch.cat([s["conv_state"].transpose(0, 1), s["x"].float()])
    y = _silu(s["b"] + sum(s["w"][j] * xp[j:j + T] for j in range(W)))
    at = n[:, None] + torch.arange(W - 1, device=DEV)
    state = xp[at, torch.arange(c["B"], device=DEV)[:, None]]
    return torch.where(valid, y.to(s["x"].dtype), s["conv_out"]), state


def _plain_scan(s, valid):
    """The recurrence h_t = a_t h_{t-1} + b_t as an inclusive scan of the pairs
    (a, b), by doubling: log2 T passes over all steps."""
    u = s["u"].float()
    d = torch.where(valid, _softplus(s["delta"].float() + s["delta_bias"]), 0.0)
    a = torch.exp(d.unsqueeze(2) * s["A"])
    b = torch.where(valid, d * u, 0.0).unsqueeze(2) * s["Bm"].float().unsqueeze(3)
    b[0] += a[0] * s["state"]
    k, T = 1, a.shape[0]
    while k < T:
        b = torch.cat([b[:k], a[k:] * b[:-k] + b[k:]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    y = (b * s["Cm"].float().unsqueeze(3)).sum(2) + s["Dskip"] * u
    y = (y * _silu(s["z"].float())).to(s["u"].dtype)
    return torch.where(valid, y, s["y"]), b[-1].clone()


def _plain(s):
    k = s["case"]["kind"]
    if k == "norm":
        return _plain_norm(s)
    if k == "grad":
        return _plain_grad(s)
    if k == "q4":
        return _plain_q4(s)
    valid, n = _valid(s["case"], s["lengths"])
    conv, conv_state = _plain_conv(s, valid, n)
    y, state = _plain_scan(s, valid)
    return dict(conv=conv, conv_state=conv_state, y=y, state=state)


# ------------------------------------------------- through the framework's calls
def _own(s):
    from paper_1607_04683_amd import qlstm as ql
    c = s["case"]
    k = c["kind"]
    if k == "norm":
        want = ("sum",) if s["residual"] is not None else ()
        if c["out"] == "y":
            return ql.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                               want=want + ("y", "rstd"))
        r = ql.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                        want=want + ("codes",))
        q = r.pop("codes")
        r["recovered"] = ql.dequantize_activations(q)
        return r
    if k == "grad":
        dx, dweight = ql.rms_norm_backward(s["dy"], s["x"], s["rstd"], s["weight"],
                                           dsum=s["residual"])
        return dict(dx=dx, dweight=dweight)
    if k == "q4":
        q = ql.QMatrix4(s["packed"], c["rows"], c["cols"], c["group"], s["zero"], s["inv_q"])
        x = s["X"] if c["x"] == "rows" else ql.QAct(s["xcodes"], c["cols"], s["xzero"],
                                                    s["xinv_q"], s["xsums"])
        return ql.matmul4(q, x, s["bias"], out_dtype=TYPES[c["type"]])
    if s["ws"] is None:
        s["ws"] = ql.Workspace()
    ql.causal_conv(s["x"], s["w"], s["b"], lengths=s["lengths"], state_in=s["conv_state"],
                   state_out=s["conv_state_out"], out=s["conv_out"])
    ql.selective_scan(s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], D=s["Dskip"], z=s["z"],
                      delta_bias=s["delta_bias"], lengths=s["lengths"], state_in=s["state"],
                      state_out=s["state_out"], out=s["y"], workspace=s["ws"])
    return dict(conv=s["conv_out"], conv_state=s["conv_state_out"], y=s["y"], state=s["state_out"])


def run(s):
    return _own(s) if own else _plain(s)


# ---------------------------------------------------------- what a pass needs
def work(case):
    c, k = case, case["kind"]
    e = 4 if c["type"] == "f32" else 2
    if k == "norm":
        n = c["m"] * c["cols"]
        reads = e * (2 if c["residual"] else 1)
        writes = (e if c["residual"] else 0) + (4 if c["out"] == "codes" else e)
        return dict(bytes=n * (reads + writes) + 4 * c["cols"], flops=8.0 * n)
    if k == "grad":
        n = c["m"] * c["cols"]
        return dict(bytes=n * e * (4 if c["residual"] else 3) + 8 * c["cols"] + 4 * c["m"],
                    flops=10.0 * n)
    if k == "q4":
        m, N, K = c["m"], c["rows"], c["cols"]
        x = m * K * (1 if c["x"] == "codes" else e)
        return dict(bytes=N * K // 2 + 5 * N * -(-K // c["group"]) + x + e * m * N,
                    flops=2.0 * m * N * K)
    T, B, D, N, W = c["T"], c["B"], c["D"], c["N"], c["W"]
    steps = T * B / 2 if c["ragged"] else T * B  # lengths lie anywhere up to T
    return dict(bytes=e * steps * (6 * D + 2 * N) + 8 * B * D * (N + W - 1) + 4 * D * (N + W + 3),
                flops=steps * D * (7.0 * N + 2 * W + 20))


# ------------------------------------------- the same values in 64-bit floats
def exact(case, seed):
    d, c, k = _draw_inputs(case, seed), case, case["kind"]
    f = lambda v: v.double()
    if k == "norm":
        v = d["x"]
        if c["residual"]:
            v = (f(d["x"]) + f(d["residual"])).to(v.dtype)
        r = torch.rsqrt(f(v).pow(2).mean(1) + EPS)
        out = dict(sum=f(v)) if c["residual"] else {}
        if c["out"] == "y":
            return dict(out, y=f(v) * r[:, None] * f(d["weight"]), rstd=r)
        # codes next to a border go by the last bit of the fp32 y: no value in 64 bits
        return dict(out, recovered=None)
    if k == "grad":
        v, dy, r, w = f(d["x"]), f(d["dy"]), f(d["rstd"])[:, None], f(d["weight"])
        xh = v * r
        dx = r * (w * dy - xh * (w * dy * xh).mean(1, keepdim=True))
        if c["residual"]:
            dx = dx + f(d["residual"])
        return dict(dx=dx, dweight=(dy * xh).sum(0))
    if k == "q4":
        rows, cols, group = c["rows"], c["cols"], c["group"]
        W, step = torch.zeros(rows, cols, dtype=torch.float64, device=DEV), 0
        for k0 in range(0, cols, group):
            w = f(d["W"][:, k0:k0 + group])
            lo, hi = w.min(1, keepdim=True)[0].clamp(max=0), w.max(1, keepdim=True)[0].clamp(min=0)
            step = torch.where(hi > lo, (hi - lo) / 15, 1.0)
            at = torch.floor(w * (15 / (15 * step)) + 0.5)
            W[:, k0:k0 + group] = at * step
        X = f(d["X"])
        lo, hi = X.min(1, keepdim=True)[0], X.max(1, keepdim=True)[0]
        step = torch.where(hi > lo, (hi - lo) / 255, 1.0)
        Y = (torch.floor(X / step + 0.5) * step) @ W.T
        return Y + f(d["bias"]) if c["bias"] else Y
    T, B, W = c["T"], c["B"], c["W"]
    n = d["lengths"].tolist() if c["ragged"] else [T] * B
    xs = torch.cat([f(d["conv_state"]).transpose(0, 1), f(d["x"])])
    acc = f(d["b"]).expand(T, B, -1).clone()
    for j in range(W):
        acc += f(d["w"][j]) * xs[j:j + T]
    conv = acc * torch.sigmoid(acc)
    conv_state = torch.stack([xs[n[b]:n[b] + W - 1, b] for b in range(B)])
    h, A = f(d["state"]).clone(), f(d["A"])
    dl = torch.logaddexp(f(d["delta"]) + f(d["delta_bias"]), torch.zeros((), dtype=torch.float64, device=DEV))
    y, at = torch.zeros(T, B, c["D"], dtype=torch.float64, device=DEV), torch.tensor(n, device=DEV)
    for t in range(T):
        on = (at > t)[:, None, None]
        dt = dl[t].unsqueeze(1)
        nh = torch.exp(dt * A) * h + dt * f(d["u"][t]).unsqueeze(1) * f(d["Bm"][t]).unsqueeze(2)
        h = torch.where(on, nh, h)
        y[t] = (h * f(d["Cm"][t]).unsqueeze(2)).sum(1)
    zz = f(d["z"])
    y = (y + f(d["Dskip"]) * f(d["u"])) * zz * torch.sigmoid(zz)
    for b in range(B):
        conv[n[b]:, b] = 0
        y[n[b]:, b] = 0
    return dict(conv=conv, conv_state=conv_state, y=y, state=h)
