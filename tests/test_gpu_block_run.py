"""A quantized state-space block run as a program runs it: norm with the residual's
addition into 8-bit codes, 4-bit in-projection, causal convolution, products
for the scan's steps, scan, 4-bit out-projection; a prompt, then single tokens
from the carried states, eager, captured into a graph, and on another stream."""
import numpy as np
import pytest
import torch

import block_reference as ref
from block_reference import f64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def ql():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_1607_04683_amd import qlstm
    qlstm.load()
    return qlstm


class Block:
    """One block: width E, D channels, N states, R columns of the step's factor."""

    def __init__(self, ql, E, D, N, R, dtype, seed):
        g = torch.Generator().manual_seed(seed)
        z = lambda *s: torch.randn(*s, generator=g).to(DEV)
        self.ql, self.E, self.D, self.N, self.R, self.dtype = ql, E, D, N, R, dtype
        self.norm = 1 + 0.1 * z(E)
        self.w_in = ql.quantize4(z(2 * D, E) * E ** -0.5, 64)
        self.conv_w, self.conv_b = 0.4 * z(4, D), 0.1 * z(D)
        self.w_x = ql.quantize4(z(R + 2 * N, D) * D ** -0.5, 32)
        self.w_dt = ql.quantize4(z(D, R) * R ** -0.5, 32)
        self.dt_bias = -4 + 0.5 * z(D)
        self.A = -torch.exp(0.5 * z(N, D))
        self.skip = z(D)
        self.w_out = ql.quantize4(z(E, D) * D ** -0.5, 128)

    def state(self, B):
        return (torch.zeros(B, 3, self.D, device=DEV), torch.zeros(B, self.N, self.D, device=DEV))

    def __call__(self, x, stream, conv, ssm, lengths=None):
        """x: what the block before it gave, stream: the residual stream (updated in place),
        both [T][B][E]; the states are updated in place -> the block's output.  What goes into
        and out of the scan stays in self.seen."""
        ql, D, N, R = self.ql, self.D, self.N, self.R
        T, B, E = x.shape
        q = ql.rms_norm(x.view(T * B, E), self.norm, residual=stream.view(T * B, E),
                        want=("sum", "codes"), out=dict(sum=stream.view(T * B, E)))["codes"]
        xz = ql.matmul4(self.w_in, q, out_dtype=self.dtype).view(T, B, 2 * D)
        u = torch.zeros(T, B, D, dtype=self.dtype, device=DEV)
        ql.causal_conv(xz[..., :D], self.conv_w, self.conv_b, lengths=lengths, state_in=conv,
                       state_out=conv, out=u)
        dbc = ql.matmul4(self.w_x, u.view(T * B, D)).view(T, B, R + 2 * N)
        delta = ql.matmul4(self.w_dt, dbc.view(T * B, R + 2 * N)[:, :R]).view(T, B, D)
        y = torch.zeros_like(u)
        ql.selective_scan(u, delta, self.A, dbc[..., R:R + N], dbc[..., R + N:], D=self.skip, z=xz[..., D:],
                          delta_bias=self.dt_bias, lengths=lengths, state_in=ssm, state_out=ssm, out=y)
        self.seen = dict(u=u, delta=delta, Bm=dbc[..., R:R + N], Cm=dbc[..., R + N:], z=xz[..., D:], y=y)
        return ql.matmul4(self.w_out, y.view(T * B, D)).view(T, B, E)

    def bounds(self, seen, lengths, state):
        """How far two evaluations of the scan, and of the block's output, may be from each
        other: (y, state, output).  The scan: twice its bound in fp32 (block_reference) and a
        step of y's type.  The output: a recovered value is within half a step of the 8-bit
        grid (range / 255) of its y, so two of them differ by a step and what y differs by;
        each counts with its weight; then the product's and the output's own rounding."""
        y, by, h, bh = ref.scan(f64(seen["u"]), f64(seen["delta"]), f64(self.A), f64(seen["Bm"]),
                                f64(seen["Cm"]), f64(self.skip), f64(seen["z"]), f64(self.dt_bias), True,
                                lengths, f64(state))
        half = ref.HALF[self.dtype]
        dy = 2 * by * (1 + half) + 2 * half * np.abs(y)
        step = (y.max(2) - y.min(2) + 2 * dy.max(2)) / 255
        W = np.abs(f64(self.ql.dequantize4(self.w_out)))
        top = np.abs(y).max(2, keepdims=True) + dy.max(2, keepdims=True) + step[..., None]
        out = dy @ W.T + step[..., None] * W.sum(1) + 2 * (half + 40 * ref.U32) * top * W.sum(1)
        return dy, 2 * bh, out


def inputs(T, B, E, dtype, seed=5):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, B, E, generator=g).to(dtype).to(DEV), torch.randn(T, B, E, generator=g).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,D,N,R", [(64, 128, 16, 8), (100, 130, 5, 7)])
def test_prompt_equals_its_tokens(ql, dtype, E, D, N, R):
    """A prompt in one call, and the same one token at a time.  Everything before the
    scan is the same bits; from there on within the bounds of its roundings."""
    T, B = 40, 3
    blk = Block(ql, E, D, N, R, dtype, 3)
    x, s = inputs(T, B, E, dtype)
    cs, hs = blk.state(B)
    s1 = s.clone()
    whole = blk(x, s1, cs, hs)
    seen = blk.seen
    cs2, hs2 = blk.state(B)
    s2, rows, parts = s.clone(), [], []
    for t in range(T):
        rows.append(blk(x[t:t + 1], s2[t:t + 1], cs2, hs2))
        parts.append(blk.seen)
    assert torch.equal(s1, s2) and torch.equal(cs, cs2)
    for k in ("u", "delta", "Bm", "Cm", "z"):
        assert torch.equal(seen[k], torch.cat([p[k] for p in parts])), k
    by, bh, bo = blk.bounds(seen, None, torch.zeros_like(hs))
    assert (np.abs(f64(seen["y"]) - f64(torch.cat([p["y"] for p in parts]))) <= by).all()
    assert (np.abs(f64(hs) - f64(hs2)) <= bh).all()
    assert (np.abs(f64(whole) - f64(torch.cat(rows))) <= bo).all()


def test_padded_batch_equals_its_sequences(ql):
    """Sequences of a padded batch, one of them empty: up to the scan the bits of each
    sequence alone, then within the bounds of its roundings."""
    E, D, N, R, T = 64, 128, 16, 8, 70
    lens = [70, 0, 1, 33, 64]
    B = len(lens)
    blk = Block(ql, E, D, N, R, torch.float32, 4)
    x, s = inputs(T, B, E, torch.float32)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    cs, hs = blk.state(B)
    cs += 0.5
    hs += 0.25
    h0 = hs.clone()
    out = blk(x, s.clone(), cs, hs, lengths=n)
    seen = blk.seen
    by, bh, bo = blk.bounds(seen, np.array(lens), h0)
    for b, L in enumerate(lens):
        c1, h1 = blk.state(1)
        c1 += 0.5
        h1 += 0.25
        o = blk(x[:L, b:b + 1].contiguous(), s[:L, b:b + 1].clone(), c1, h1)
        assert torch.equal(cs[b:b + 1], c1)
        for k in ("u", "delta", "Bm", "Cm", "z"):
            assert torch.equal(seen[k][:L, b], blk.seen[k][:, 0]), k
        assert (np.abs(f64(hs[b:b + 1]) - f64(h1)) <= bh[b]).all()
        assert not seen["y"][L:, b].any()
        assert (np.abs(f64(seen["y"][:L, b]) - f64(blk.seen["y"][:, 0])) <= by[:L, b]).all()
        assert (np.abs(f64(out[:L, b]) - f64(o[:, 0])) <= bo[:L, b]).all()


def test_tokens_from_a_graph(ql):
    """A token's step captured and replayed, with eager steps of another block between
    the replays: the bits of eager steps.  The second graph has its own memory."""
    E, D, N, R, B = 128, 256, 16, 8, 2
    blk, other = Block(ql, E, D, N, R, torch.bfloat16, 6), Block(ql, E, D, N, R, torch.bfloat16, 7)
    T = 6
    x, s = inputs(T, B, E, torch.bfloat16)
    cs, hs = blk.state(B)
    want, states = [], []
    for t in range(T):
        want.append(blk(x[t:t + 1], s[t:t + 1].clone(), cs, hs))
        states.append((cs.clone(), hs.clone()))
    gx, gs = x[:1].clone(), s[:1].clone()
    graphs = []
    for _ in range(2):
        c, h = blk.state(B)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            blk(gx, gs.clone(), c, h)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = blk(gx, gs, c, h)
        graphs.append((g, c, h, o))
        c.zero_()
        h.zero_()
    for t in range(T):
        for g, c, h, o in graphs:
            gx.copy_(x[t:t + 1])
            gs.copy_(s[t:t + 1])
            g.replay()
            c2, h2 = other.state(B)
            other(x[t:t + 1], s[t:t + 1].clone(), c2, h2)
            torch.cuda.synchronize()
            assert torch.equal(o, want[t]), t
            assert torch.equal(c, states[t][0]) and torch.equal(h, states[t][1]), t


def test_two_streams_at_once(ql):
    """Two prompts on two streams, each with its own workspace: the bits of one after the other."""
    E, D, N, R, T, B = 64, 192, 16, 8, 300, 1
    blk = Block(ql, E, D, N, R, torch.float32, 8)
    xs = [inputs(T, B, E, torch.float32, seed=k) for k in (1, 2)]
    want = []
    for x, s in xs:
        c, h = blk.state(B)
        want.append((blk(x, s.clone(), c, h), c, h))
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    states = [blk.state(B) for _ in xs]
    copies = [s.clone() for _, s in xs]
    torch.cuda.synchronize()
    for st, (x, _), (c, h), s in zip(streams, xs, states, copies):
        with torch.cuda.stream(st):
            got.append((blk(x, s, c, h), c, h))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_norm_gradients_of_a_stack(ql):
    """Two norms on one residual stream, forward and backward through the framework's calls,
    against autograd in 64 bits on the CPU.  Each fp32 gradient passes two norms' chains
    of some 40 roundings: 200 half steps of the largest gradient of the row."""
    m, n, eps = 50, 300, 1e-6
    g = torch.Generator().manual_seed(1)
    z = lambda *s: torch.randn(*s, generator=g)
    x, r, w1, w2, dy1, dy2 = z(m, n), z(m, n), 1 + 0.1 * z(n), 1 + 0.1 * z(n), z(m, n), z(m, n)
    d = lambda t: t.to(DEV)
    a = ql.rms_norm(d(x), d(w1), residual=d(r), eps=eps, want=("y", "sum", "rstd"))
    b = ql.rms_norm(a["y"], d(w2), residual=a["sum"], eps=eps, want=("y", "sum", "rstd"))
    ds2, dw2 = ql.rms_norm_backward(d(dy2), b["sum"], b["rstd"], d(w2))
    # the second stream is y1 + stream 1: its gradient arrives at both
    ds1, dw1 = ql.rms_norm_backward(ds2 + d(dy1), a["sum"], a["rstd"], d(w1), dsum=ds2)
    p = [t.double().requires_grad_() for t in (x, r, w1, w2)]
    v1 = p[0] + p[1]
    y1 = v1 * torch.rsqrt(v1.square().mean(1, keepdim=True) + eps) * p[2]
    v2 = y1 + v1
    y2 = v2 * torch.rsqrt(v2.square().mean(1, keepdim=True) + eps) * p[3]
    ((y1 * dy1.double()).sum() + (y2 * dy2.double()).sum()).backward()
    for got, want in ((ds1, p[0].grad), (ds1, p[1].grad), (dw1, p[2].grad), (dw2, p[3].grad)):
        e = (got.cpu().double() - want).abs().max()
        assert e <= 200 * 2.0 ** -24 * want.abs().max(), e
