"""The operators around the attention together, as a backbone layer uses them.

Serving: a qkv projection with 4-bit weights, norm and rotation of its heads into the attention's E4M3 form, the attention.
Training: the FP8 layer that keeps 8 bits of its input, norm and rotation, and the gradients of both, back to x, W, the bias and the
norm's parameters."""
import numpy as np
import pytest
import torch

from oracle import projection_oracle as po
from paper_2605_11354_amd import binding as B
from paper_2605_11354_amd import synth
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
f64 = G.bf16_tensor_to_f64


def draw(seed, N, d_in, d_out):
    g = np.random.default_rng(seed)
    bits = lambda a: synth.to_bf16_bits(a.astype(np.float32))
    return g, bits(g.standard_normal((N, d_in))), bits(g.standard_normal((d_out, d_in)) / np.sqrt(d_in)), bits(0.1 * g.standard_normal(d_out))


@pytest.mark.parametrize("Bn,N,H,bq", [(1, 700, 2, 128), (3, 130, 4, 64), (5, 1, 2, 64)])
def test_serving_layer(oracle, Bn, N, H, bq):
    d_in, D = 128 * H, 64
    g, xb, Wb, bb = draw(N, Bn * N, d_in, 3 * H * D)
    x, W, bias = map(G.dev_bf16, (xb, Wb, bb))
    Wc, Ws = torch.empty((3 * H * D, d_in // 2), dtype=torch.uint8, device="cuda"), torch.empty((3 * H * D, d_in // 32), dtype=torch.uint8, device="cuda")
    B.sla_quantise_mxfp4(W, Wc, Ws)
    qkv = torch.empty((Bn * N, 3 * H * D), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.view(Bn, N, 3, H, D).unbind(2)
    hp = B.make_heads_params(q, norm="layer", axes=2, base=100.0, layout="bnhd")
    pos = torch.from_numpy(g.integers(0, 40, (N, 2)).astype(np.int32)).cuda()
    w = [torch.from_numpy((1 + 0.1 * g.standard_normal(64)).astype(np.float32)).cuda() for _ in range(2)]
    codes = [torch.empty((Bn, N, H, D), dtype=torch.uint8, device="cuda") for _ in range(3)]
    scales = [torch.empty((Bn, H, -(-N // b)), device="cuda") for b in (bq, 64, 64)]
    O = torch.empty((Bn, N, H, D), dtype=torch.bfloat16, device="cuda")
    Wp = G.dev_bf16(synth.to_bf16_bits((g.standard_normal((D, D)) / 8).astype(np.float32)))
    nkb = -(-N // 64)
    p = B.make_params(Bn, H, N, bq, 64, 0.0, 0.0, max(1, nkb // 3), nkb // 4, "fp8", False, layout="bnhd")
    ws, mws = B.alloc_workspace(p), torch.empty(max(256, B.sla_mxfp4_linear_workspace_bytes(Bn * N, d_in, 3 * H * D)), dtype=torch.uint8, device="cuda")

    def layer():
        B.sla_mxfp4_linear(x, Wc, Ws, bias, qkv, mws)
        B.sla_qk_norm_rope_e4m3(hp, q, k, v, bq, *codes, *scales, pos=pos, q_weight=w[0], k_weight=w[1])
        B.sla_forward(p, *codes, Wp, O, None, *scales, ws)

    layer()
    torch.cuda.synchronize()
    # the projection, against exact products of the 4-bit numbers
    xq, wq = po.mxfp4_values(*po.mxfp4_quantise(xb)), po.mxfp4_values(*po.mxfp4_quantise(Wb))
    ref = xq @ wq.T + po.bf16_to_f64(bb)
    assert (np.abs(f64(qkv) - ref) <= 2.0 ** -8 * np.abs(ref) + (d_in + 2) * 2.0 ** -24 * (np.abs(xq) @ np.abs(wq).T + np.abs(po.bf16_to_f64(bb)))).all()
    # the heads, from the projection's own bf16 values: half an E4M3 step (and 1e-5 of the largest for the fp32 arithmetic in front)
    rows = f64(qkv).reshape(Bn, N, 3, H, D)
    for n, (c, s, blk) in enumerate(zip(codes, scales, (bq, 64, 64))):
        y = rows[:, :, n] if n == 2 else po.heads_forward(rows[:, :, n], "layer", w[n].double().cpu().numpy(), None, 1e-5, 2, "halves", 100.0, pos.cpu().numpy())
        sc = np.repeat(s.double().cpu().numpy().transpose(0, 2, 1), blk, 1)[:, :N, :, None]
        got = c.view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64) * sc
        assert (np.abs(got - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * sc + 1e-5 * np.abs(y).max()).all(), n
    # the attention, from the codes it was given, against the oracle (head-major there)
    hm = lambda t: np.ascontiguousarray(t.cpu().numpy().transpose(0, 2, 1, 3))
    kc, kn = B.sla_resolve_counts(p)
    op = oracle.make_params(Bn, H, N, bq, 64, kc, kn, "fp8", False)
    want = oracle.forward(op, *(hm(c) for c in codes), Wp.view(torch.int16).cpu().numpy().view(np.uint16)[None], *(s.cpu().numpy() for s in scales))["O"]
    G.assert_output(f64(O).transpose(0, 2, 1, 3), want, "fp8", "serving layer")
    # and all of it from one captured graph, several times
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for r in range(3):
        x.mul_(1.25)
        layer()
        torch.cuda.synchronize()
        eager = O.clone()
        O.zero_(), qkv.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.view(torch.int16), O.view(torch.int16)), r


@pytest.mark.parametrize("Bn,N,H,per_head", [(1, 300, 3, False), (2, 65, 4, True), (4, 1, 2, False)])
def test_training_layer(Bn, N, H, per_head):
    """Against the same chain in fp64.  Each bf16 store is a relative error of at most 2^-8 / sqrt(3) in the 2-norm; qkv, dqkv, x_q or W_q
    and the result make four of them, each of which reaches the result with a factor of about one (a norm's Jacobian keeps the size of a
    perturbation relative to its row): 4 * 2.3e-3 at most, and half of that if they were independent."""
    d_in, D, T = 128 * H, 64, Bn * N
    g, xb, Wb, bb = draw(7 + N, T, d_in, 3 * H * D)
    x, W, bias = map(G.dev_bf16, (xb, Wb, bb))
    qkv, dqkv = torch.empty((T, 3 * H * D), dtype=torch.bfloat16, device="cuda"), torch.full((T, 3 * H * D), float("nan"), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.view(Bn, N, 3, H, D).unbind(2)
    dq, dk, dv = dqkv.view(Bn, N, 3, H, D).unbind(2)
    hp = B.make_heads_params(q, norm="rms", norm_per_head=per_head, axes=1, pairing="adjacent", base=1e4, pos_per_item=True)
    pos = torch.from_numpy(g.integers(0, 5000, (Bn, N, 1)).astype(np.int32)).cuda()
    shape = (H, 64) if per_head else (64,)
    w = [torch.from_numpy((1 + 0.2 * g.standard_normal(shape)).astype(np.float32)).cuda() for _ in range(2)]
    out, grads = ([torch.empty((Bn, H, N, D), dtype=torch.bfloat16, device="cuda") for _ in range(3)] for _ in range(2))
    for t in grads:
        t.copy_(torch.from_numpy(g.standard_normal(t.shape).astype(np.float32)))
    ck = torch.empty(B.sla_fp8_checkpoint_bytes(T, d_in), dtype=torch.uint8, device="cuda")
    dw = [torch.empty(shape, device="cuda") for _ in range(2)]
    dx, dW, db = torch.empty_like(x), torch.empty_like(W), torch.empty_like(bias)

    B.sla_fp8_linear_save(x, W, bias, qkv, ck)
    B.sla_qk_norm_rope(hp, q, k, v, *out, pos=pos, q_weight=w[0], k_weight=w[1])
    x.fill_(float("nan"))                             # the input is free from here on
    B.sla_qk_norm_rope_grad(hp, q, k, *grads, dq, dk, dv, pos=pos, q_weight=w[0], k_weight=w[1], dq_weight=dw[0], dk_weight=dw[1])
    B.sla_fp8_linear_grad(dqkv, ck, W, dx, dW, db)
    torch.cuda.synchronize()

    y = po.fp8_linear_train(xb, Wb, bb).reshape(Bn, N, 3, H, D)
    rot = (1, "adjacent", 1e4, pos.cpu().numpy())
    d = np.empty_like(y)
    for n in range(3):
        gy = f64(grads[n]).transpose(0, 2, 1, 3)
        if n == 2:
            d[:, :, 2] = gy
            continue
        wn = w[n].double().cpu().numpy()
        fwd = po.heads_forward(y[:, :, n], "rms", wn, None, 1e-5, *rot)
        assert np.linalg.norm(f64(out[n]).transpose(0, 2, 1, 3) - fwd) <= 4.7e-3 * np.linalg.norm(fwd)           # two stores
        d[:, :, n], rw, _ = po.heads_backward(y[:, :, n], "rms", wn, 1e-5, *rot, gy, per_head=per_head)
        assert np.linalg.norm(dw[n].double().cpu().numpy() - rw) <= 2.4e-3 * np.linalg.norm(rw) + 1e-6           # one store, of qkv
    rx, rW, rb = po.fp8_linear_backward(xb, Wb, d.reshape(T, -1))
    for got, ref in ((dx, rx), (dW, rW), (db, rb)):
        assert np.linalg.norm(f64(got) - ref) <= 9.4e-3 * np.linalg.norm(ref)


def test_calls_at_once_on_two_streams():
    """Two layers on two streams, each with workspaces of its own: the bits of one after the other."""
    def make(seed, N, d_in, H):
        g, xb, Wb, bb = draw(seed, N, d_in, 3 * H * 64)
        t = dict(x=G.dev_bf16(xb), W=G.dev_bf16(Wb), b=G.dev_bf16(bb), N=N, H=H, d_in=d_in, d_out=3 * H * 64)
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
        t.update(y=bf(N, t["d_out"]), ck=u8(B.sla_fp8_checkpoint_bytes(N, d_in)), ws=u8(B.sla_fp8_linear_grad_workspace_bytes(N, d_in, t["d_out"])),
                 dx=bf(N, d_in), dW=bf(t["d_out"], d_in), db=bf(t["d_out"]), Wc=u8(t["d_out"], d_in // 2), Ws=u8(t["d_out"], d_in // 32), y4=bf(N, t["d_out"]),
                 mws=u8(max(256, B.sla_mxfp4_linear_workspace_bytes(N, d_in, t["d_out"]))), out=[bf(1, H, N, 64) for _ in range(3)], d=bf(N, t["d_out"]),
                 dw=[torch.zeros(64, device="cuda") for _ in range(4)])
        t["p"] = B.make_heads_params(t["y"].view(1, N, 3, H, 64)[:, :, 0], axes=0)
        t["hws"] = u8(max(256, B.sla_qk_norm_rope_grad_workspace_bytes(t["p"])))
        return t

    def layer(t):
        B.sla_fp8_linear_save(t["x"], t["W"], t["b"], t["y"], t["ck"], t["ws"])
        q, k, v = t["y"].view(1, t["N"], 3, t["H"], 64).unbind(2)
        B.sla_qk_norm_rope(t["p"], q, k, v, *t["out"])
        d = t["d"].view(1, t["N"], 3, t["H"], 64).unbind(2)
        B.sla_qk_norm_rope_grad(t["p"], q, k, *t["out"], *d, dq_weight=t["dw"][0], dq_bias=t["dw"][1], dk_weight=t["dw"][2], dk_bias=t["dw"][3], workspace=t["hws"])
        B.sla_fp8_linear_grad(t["d"], t["ck"], t["W"], t["dx"], t["dW"], t["db"], t["ws"])
        B.sla_quantise_mxfp4(t["W"], t["Wc"], t["Ws"])
        B.sla_mxfp4_linear(t["x"], t["Wc"], t["Ws"], t["b"], t["y4"], t["mws"])
        return [t["y"], *t["out"], t["d"], *t["dw"], t["dx"], t["dW"], t["db"], t["y4"]]

    layers = make(1, 1500, 384, 4), make(2, 700, 512, 6)
    want = [[o.clone() for o in layer(t)] for t in layers]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for t, s in zip(layers, streams):
            with torch.cuda.stream(s):
                for name in ("y", "dx", "dW", "db", "y4", "d"):
                    t[name].zero_()
                got.append(layer(t))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
