"""Norm and rotation of heads against the fp64 reference, through the binding.

Tolerances.  u = 2^-24 is half a step of fp32.  A row's mean takes 9 roundings and its square sum 11, the divisions and the
root 4, the weights and the bias 2, the rotation 4 with angles that are exact to 2^-23 of a turn (and sincospi's few u): an
output is off by at most 64 u (A + X) with A the largest |n| and X the largest |x| r |w| of the row (what the subtraction of
the mean loses), before half a bf16 step, 2^-8 relative to the result.  Backward: dx carries two more sums of the same length
over products with |u| <= 8, at most 512 u r G (1 + X) with G the row's largest |g|."""
import numpy as np
import pytest
import torch

from oracle import projection_oracle as po
from paper_2605_11354_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
f64 = lambda t: t.detach().float().cpu().numpy().astype(np.float64)


def sources(kind, Bn, N, H, pad=0):
    """q, k, v as views [B,N,H,64] of a buffer, and the buffer."""
    if kind == "fused":
        t = torch.full((Bn, N, 3, H, 64 + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        return t, [t[:, :, i, :, :64] for i in range(3)]
    if kind == "per_head":
        t = torch.full((Bn, N, H, 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        return t, [t[:, :, :, i] for i in range(3)]
    if kind == "token_first":
        t = torch.full((N, Bn, 3, H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        return t, [t[:, :, i].transpose(0, 1) for i in range(3)]
    t = torch.full((3, Bn, H, N, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    return t, [t[i].transpose(1, 2) for i in range(3)]


class Heads:
    def __init__(self, Bn, N, H, norm="layer", per_head=False, axes=2, pairing="halves", base=100.0, kind="fused", layout="bhnd",
                 own_pos=False, seed=0, far=0, pad=0, weights=True):
        g = np.random.default_rng(seed)
        self.B, self.N, self.H, self.norm, self.per_head, self.layout, self.kind, self.pad = Bn, N, H, norm, per_head, layout, kind, pad
        self.buf, self.x = sources(kind, Bn, N, H, pad)
        for t in self.x:
            level = np.exp(g.uniform(-2, 2, (Bn, N, H, 1)))
            t.copy_(torch.from_numpy((level * (g.standard_normal((Bn, N, H, 64)) + g.standard_normal((Bn, N, H, 1)))).astype(np.float32)))
        shape = (H, 64) if per_head else (64,)
        par = lambda at: torch.from_numpy((at + 0.3 * g.standard_normal(shape)).astype(np.float32)).cuda() if norm != "none" and weights else None
        self.w, self.b = [par(1.0), par(1.0)], [par(0.0), par(0.0)]
        self.pos = None
        if axes:
            pos = g.integers(-far - 40, far + 40, (Bn if own_pos else 1, N, axes))
            self.pos = torch.from_numpy(pos.astype(np.int32)).cuda()
        self.p = B.make_heads_params(self.x[0], norm, per_head, 1e-5, axes, pairing, base, own_pos, layout)
        self.rot = (axes, pairing, base, None if self.pos is None else self.pos.cpu().numpy())
        self.kw = dict(pos=self.pos, q_weight=self.w[0], k_weight=self.w[1])
        self.bias = dict(q_bias=self.b[0], k_bias=self.b[1])

    def out(self, dtype=torch.bfloat16, fill=float("nan")):
        shape = (self.B, self.N, self.H, 64) if self.layout == "bnhd" else (self.B, self.H, self.N, 64)
        return [torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(3)]

    def bnhd(self, t):
        return t if self.layout == "bnhd" else t.transpose(1, 2)

    def reference(self, n):
        """(y [B,N,H,64], what it may be off by before the last rounding)."""
        x = f64(self.x[n])
        if n == 2:
            return x, np.zeros_like(x[..., :1])
        w, b = (None if t[n] is None else f64(t[n]) for t in (self.w, self.b))
        y = po.heads_forward(x, self.norm, w, b, 1e-5, *self.rot)
        u, r = po._unit(x, self.norm, 1e-5)
        n_ = np.abs(u * (1 if w is None else w)) + (0 if b is None else np.abs(b))
        loss = np.abs(x).max(-1, keepdims=True) * (1 if r is None else r) * (1 if w is None else np.abs(w).max())
        return y, 64 * U * (n_.max(-1, keepdims=True) + loss)

    def forward(self, v=True):
        Q, K, V = self.out()
        B.sla_qk_norm_rope(self.p, *self.x[:2], self.x[2] if v else None, Q, K, V if v else None, **self.kw, **self.bias)
        torch.cuda.synchronize()
        return [Q, K, V] if v else [Q, K]

    def check_forward(self, got):
        for n, t in enumerate(got):
            y, off = self.reference(n)
            d = np.abs(f64(self.bnhd(t)) - y)
            assert (d <= 2.0 ** -8 * np.abs(y) + off).all(), (n, d.max(), np.nanmax(d / (2.0 ** -8 * np.abs(y) + off + 1e-300)))


CASES = [
    dict(Bn=1, N=1, H=1), dict(Bn=3, N=1, H=16, norm="rms", axes=1, pairing="adjacent", base=1e6, own_pos=True, far=2 ** 31 - 41),
    dict(Bn=1, N=64, H=4), dict(Bn=1, N=65, H=5, norm="rms", kind="per_head", layout="bnhd"), dict(Bn=2, N=63, H=3, per_head=True, own_pos=True),
    dict(Bn=5, N=37, H=7, axes=1, base=1e4, kind="head_major", far=100000), dict(Bn=2, N=129, H=2, axes=2, pairing="adjacent", layout="bnhd", pad=8),
    dict(Bn=1, N=200, H=3, norm="none", axes=2), dict(Bn=1, N=130, H=12, norm="layer", axes=0, per_head=True), dict(Bn=1, N=70, H=2, norm="none", axes=0),
    dict(Bn=1, N=4500, H=16, kind="per_head"), dict(Bn=70, N=2, H=1, axes=1, own_pos=True), dict(Bn=2, N=100, H=6, weights=False),
    dict(Bn=3, N=75, H=2, kind="token_first"), dict(Bn=3, N=11003, H=2), dict(Bn=1, N=33001, H=1, norm="rms", axes=1, pairing="adjacent", base=1e4, layout="bnhd"),
]


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    h = Heads(**case)
    before = h.buf.clone()
    h.check_forward(h.forward())
    assert torch.equal(h.buf.view(torch.int16), before.view(torch.int16))


def test_forward_without_v_and_with_one_weight():
    h = Heads(2, 77, 3)
    h.w[1] = h.b[0] = None
    h.kw["k_weight"] = h.bias["q_bias"] = None
    h.check_forward(h.forward(v=False))


@pytest.mark.parametrize("bq", [64, 128])
@pytest.mark.parametrize("case", CASES)
def test_e4m3(case, bq):
    """Codes: half a step of E4M3 (2^-4 relative, 2^-10 of the scale below its normal range) from the values."""
    h = Heads(**case)
    codes = h.out(torch.uint8, 0x55)
    scales = [torch.full((h.B, h.H, -(-h.N // blk) + 1), float("nan"), device="cuda") for blk in (bq, 64, 64)]
    tight = [s.reshape(-1)[: h.B * h.H * (s.shape[2] - 1)].view(h.B, h.H, -1) for s in scales]
    B.sla_qk_norm_rope_e4m3(h.p, *h.x, bq, *codes, *tight, **h.kw, **h.bias)
    torch.cuda.synchronize()
    for n, (c, s, blk) in enumerate(zip(codes, tight, (bq, 64, 64))):
        y, off = h.reference(n)
        pad = np.zeros((h.B, -h.N % blk, h.H, 64))
        top = np.concatenate([np.abs(y), pad], 1).reshape(h.B, -1, blk, h.H, 64).max((2, 4))
        most = np.concatenate([off + 0 * y, pad], 1).reshape(h.B, -1, blk, h.H, 64).max((2, 4))
        want = np.maximum(top, 1e-8).transpose(0, 2, 1) / 448.0
        got = f64(s)
        assert (np.abs(got - want) <= 2 * U * want + most.transpose(0, 2, 1) / 448.0).all()
        sc = np.repeat(got.transpose(0, 2, 1), blk, 1)[:, : h.N, :, None]
        val = f64(h.bnhd(c).contiguous().view(torch.float8_e4m3fn)) * sc
        assert (np.abs(val - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * sc + 1.07 * off + 8 * U * np.abs(y)).all(), n
    if h.N > 0:                                       # V is the stand-alone quantiser's, bit for bit
        v = h.x[2].contiguous() if h.layout == "bnhd" else h.x[2].transpose(1, 2).contiguous()
        c2, s2 = torch.empty_like(codes[2]), torch.empty_like(tight[2].contiguous())
        B.sla_quantise_e4m3(v, 64, c2, s2, layout=h.layout)
        torch.cuda.synchronize()
        assert torch.equal(c2, codes[2]) and torch.equal(s2, tight[2])


@pytest.mark.parametrize("case", CASES)
def test_gradients(case):
    h = Heads(**case)
    g = [t.copy_(torch.from_numpy((0.01 * np.random.default_rng(9 + i).standard_normal(t.shape)).astype(np.float32))) for i, t in enumerate(h.out())]
    dbuf, dx = sources(h.kind, h.B, h.N, h.H, h.pad)
    shape = (h.H, 64) if h.per_head else (64,)
    dw = [torch.full(shape, float("nan"), device="cuda") if h.norm != "none" else None for _ in range(4)]
    names = ("dq_weight", "dq_bias", "dk_weight", "dk_bias")
    call = lambda: B.sla_qk_norm_rope_grad(h.p, *h.x[:2], *g, *dx, **h.kw, **dict(zip(names, dw)))
    call()
    torch.cuda.synchronize()
    first = [t.clone() for t in dx] + [t.clone() for t in dw if t is not None]
    for n in range(3):
        dy, x = f64(h.bnhd(g[n])), f64(h.x[n])
        if n == 2:
            assert np.array_equal(f64(dx[2]), dy)
            continue
        w = None if h.w[n] is None else f64(h.w[n])
        ref, rw, rb = po.heads_backward(x, h.norm, w, 1e-5, *h.rot, dy, per_head=h.per_head)
        u, r = po._unit(x, h.norm, 1e-5)
        r = np.ones_like(x[..., :1]) if r is None else r
        G = np.sqrt(2.0) * np.abs(dy).max(-1, keepdims=True) * (1 if w is None else np.abs(w).max())
        X = np.abs(x).max(-1, keepdims=True) * r
        d = np.abs(f64(dx[n]) - ref)
        assert (d <= 2.0 ** -8 * np.abs(ref) + 512 * U * r * G * (1 + X)).all(), (n, d.max())
        if rw is None:
            continue
        # sums: 8 rows of a unit, its units, 3 steps over lanes, 4 waves, the slots: at most the number of rows a lane adds + 80
        over, depth = ((0, 1) if h.per_head else (0, 1, 2)), 8 * (1 if h.per_head else 3 * h.H) + h.B * h.N / 64 / 64 * 24 + 80
        turned = np.abs(po._turn(dy, *h.rot[:1], h.rot[2], h.rot[1], h.rot[3], back=True)) + 8 * U * G
        bound_w = (depth * U * (turned * np.abs(u)) + 64 * U * G * (1 + X + np.abs(u))).sum(over)
        bound_b = (depth * U * turned + 16 * U * G).sum(over)
        assert (np.abs(f64(dw[2 * n]) - rw) <= bound_w).all() and (np.abs(f64(dw[2 * n + 1]) - rb) <= bound_b).all(), n
    if h.pad:                                         # what lies between the rows is left as it was
        assert bool((dbuf[..., 64:] == 7.0).all())
    for t in dx:
        t.zero_()
    call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, dx + [t for t in dw if t is not None]))


def test_gradients_of_some_parameters_and_of_no_tokens():
    h = Heads(2, 50, 3)
    g, (_, dx) = h.out(fill=0.5), sources("fused", 2, 50, 3)
    full, one = [torch.empty(64, device="cuda") for _ in range(4)], torch.empty(64, device="cuda")
    B.sla_qk_norm_rope_grad(h.p, *h.x[:2], g[0], g[1], None, dx[0], dx[1], None, **h.kw, dq_weight=full[0], dq_bias=full[1], dk_weight=full[2], dk_bias=full[3])
    B.sla_qk_norm_rope_grad(h.p, *h.x[:2], g[0], g[1], None, dx[0], dx[1], None, **h.kw, dk_weight=one)
    none = B.make_heads_params(h.x[0][:, :0])
    e = h.x[0][:, :0]
    z = torch.empty((2, 3, 0, 64), dtype=torch.bfloat16, device="cuda")
    zero = torch.full((64,), 3.0, device="cuda")
    B.sla_qk_norm_rope_grad(none, e, e, z, z, None, e, e, None, dq_bias=zero)
    torch.cuda.synchronize()
    assert torch.equal(one, full[2]) and bool((zero == 0).all())


def test_rows_of_zeros_infinities_and_nan_stay_by_themselves():
    h = Heads(1, 70, 2)
    h.x[0][0, 3, 1] = 0.0
    clean = h.forward()
    y, off = h.reference(0)
    assert (np.abs(f64(clean[0])[0, 1, 3] - y[0, 3, 1]) <= 2.0 ** -8 * np.abs(y[0, 3, 1]) + off[0, 3, 1]).all()
    h.x[0][0, 5, 0, 7], h.x[1][0, 69, 1, 0] = float("inf"), float("nan")
    got = h.forward()
    assert torch.isnan(got[0][0, 0, 5]).all() and torch.isnan(got[1][0, 1, 69]).all()
    for t, n, i in ((0, 0, 5), (1, 1, 69)):
        got[t][0, n, i] = clean[t][0, n, i]
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(clean, got))


def test_replays_from_a_graph_on_another_stream():
    h = Heads(2, 333, 4, per_head=False, own_pos=True)
    g, (_, dx) = h.out(fill=0.25), sources("fused", 2, 333, 4)
    Q, K, V = h.out()
    dw = [torch.zeros(64, device="cuda") for _ in range(4)]
    ws = torch.empty(B.sla_qk_norm_rope_grad_workspace_bytes(h.p), dtype=torch.uint8, device="cuda")

    def work():
        B.sla_qk_norm_rope(h.p, *h.x, Q, K, V, **h.kw, **h.bias)
        B.sla_qk_norm_rope_grad(h.p, *h.x[:2], *g, *dx, **h.kw, dq_weight=dw[0], dq_bias=dw[1], dk_weight=dw[2], dk_bias=dw[3], workspace=ws)

    outs = [Q, K, V, *dx, *dw]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        work()
    for k in range(3):
        h.x[0].mul_(1.0 + k), g[1].add_(0.125)
        work()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), k


def test_tensors_of_another_shape_type_or_place_are_refused():
    h = Heads(2, 5, 3)
    out, bad = h.out(), torch.empty(32, device="cuda")
    pos = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype, device="cuda")
    for name, kw in [("q_weight", dict(q_weight=bad)), ("k_bias", dict(k_bias=torch.empty(64))), ("pos", dict(pos=pos(5, 1))), ("pos", dict(pos=pos(2, 5, 2))),
                     ("pos", dict(pos=pos(5, 2, dtype=torch.int64)))]:
        with pytest.raises(ValueError, match=name):
            B.sla_qk_norm_rope(h.p, *h.x, *out, **kw)
    with pytest.raises(ValueError, match="K: "):
        B.sla_qk_norm_rope(h.p, *h.x, out[0], out[1][:, :, :4], out[2], pos=h.pos)
    with pytest.raises(ValueError, match="k: "):
        B.sla_qk_norm_rope(h.p, h.x[0], h.x[1].float(), h.x[2], *out, pos=h.pos)
    h.p.pos_per_item = 1
    with pytest.raises(ValueError, match="pos"):                                             # two items, positions of one
        B.sla_qk_norm_rope(h.p, *h.x, *out, pos=h.pos)


@pytest.mark.parametrize("bq", [64, 128])
def test_e4m3_of_infinities_and_nan_is_the_quantiser_s(bq):
    """Without norm and rotation q and k are quantised as they are: a block with an infinity (or of NaN alone) comes out as
    sla_quantise_e4m3 leaves it, v bit for bit, q and k in scales and in which values are finite."""
    h = Heads(2, 300, 3, norm="none", axes=0)
    for t in h.x:
        t[0, 5, 0, 7], t[1, 70, 1, 0], t[1, 299, 2, 63] = float("inf"), float("nan"), float("-inf")
        t[0, 128:192, 2] = float("nan")
    codes = [torch.empty((2, 3, 300, 64), dtype=torch.uint8, device="cuda") for _ in range(3)]
    scales = [torch.empty((2, 3, -(-300 // b)), device="cuda") for b in (bq, 64, 64)]
    B.sla_qk_norm_rope_e4m3(h.p, *h.x, bq, *codes, *scales)
    for n, blk in enumerate((bq, 64, 64)):
        c, s = torch.empty_like(codes[n]), torch.empty_like(scales[n])
        B.sla_quantise_e4m3(h.x[n].transpose(1, 2).contiguous(), blk, c, s)
        torch.cuda.synchronize()
        assert torch.equal(s, scales[n]) and (n < 2 or torch.equal(c, codes[n]))
        got, want = (t.view(torch.float8_e4m3fn).float() * s.repeat_interleave(blk, 2)[:, :, :300, None] for t in (codes[n], c))
        assert torch.equal(got.isfinite(), want.isfinite())
        # a product with 1 / scale instead of the quotient: the neighbouring code where the quotient lies half-way, a step of 2^-3
        ok = want.isfinite()
        assert bool(((got - want).abs()[ok] <= 2.0 ** -3 * want.abs()[ok] + 2.0 ** -9 * s.repeat_interleave(blk, 2)[:, :, :300, None].expand_as(want)[ok]).all())
