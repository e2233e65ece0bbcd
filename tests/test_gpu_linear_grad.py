"""The FP8 layer's training step from the 8-bit copy of its input, against the fp64 reference.

Tolerances.  x_q and W_q are code x scale rounded in fp32 (2^-24 relative) and to bf16 (2^-8 of the value at most, so is dy's half of the
product untouched): |error of a sum over k| <= (2^-8 + (K + 20) 2^-24) sum |dy| |q| before half a bf16 step, 2^-8 of the result.  The sum
of magnitudes is a worst case; the 2-norm of the error over a whole output, which averages the roundings, is bounded by
2^-8 / sqrt(3) for the values and as much for the store: together 2^-8 sqrt(2/3) < 3.2e-3 of the result's."""
import numpy as np
import pytest
import torch

from oracle import projection_oracle as po
from paper_2605_11354_amd import binding as B
from paper_2605_11354_amd import synth
from tests import gpu_util as G

pytestmark = pytest.mark.gpu
f64 = G.bf16_tensor_to_f64


def layer(N, d_in, d_out, seed=0):
    g = np.random.default_rng(seed)
    x = synth.to_bf16_bits((g.standard_normal((N, d_in)) * np.exp(g.uniform(-2, 2, (N, 1)))).astype(np.float32))
    W = synth.to_bf16_bits((g.standard_normal((d_out, d_in)) / np.sqrt(d_in)).astype(np.float32))
    b = synth.to_bf16_bits(g.standard_normal(d_out).astype(np.float32))
    dy = synth.to_bf16_bits((0.01 * g.standard_normal((N, d_out)) * np.exp(g.uniform(-2, 2, (N, 1)))).astype(np.float32))
    return x, W, b, dy


def buffers(N, d_in, d_out):
    ck = torch.full((B.sla_fp8_checkpoint_bytes(N, d_in) + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    ws = torch.full((B.sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out) + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    nan = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")
    return ck, ws, nan(N, d_out), nan(N, d_in), nan(d_out, d_in), nan(d_out)


def check(got, ref, mag, K, what):
    d = np.abs(got - ref)
    assert (d <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + (K + 20) * 2.0 ** -24) * mag).all(), (what, d.max())
    assert np.linalg.norm(got - ref) <= 3.2e-3 * np.linalg.norm(ref) + 1e-30 or ref.size < 64, what


SIZES = [(1, 128, 8), (33, 256, 72), (64, 384, 136), (31, 128, 264), (197, 384, 1152), (1000, 128, 64), (2049, 640, 520), (4099, 256, 2056), (300, 1152, 4104)]


@pytest.mark.parametrize("N,d_in,d_out", SIZES)
def test_training_step(N, d_in, d_out):
    x, W, b, dy = layer(N, d_in, d_out, N)
    X, Wd, bd, dyd = map(G.dev_bf16, (x, W, b, dy))
    ck, ws, y, dx, dW, db = buffers(N, d_in, d_out)
    B.sla_fp8_linear_save(X, Wd, bd, y, ck[:-256], ws[:-256])
    kept = ck.clone()
    X.zero_()                                         # the backward pass has the 8-bit copy alone
    ws[:-256] = 0xFF                                  # and a workspace that holds nothing
    B.sla_fp8_linear_grad(dyd, ck[:-256], Wd, dx, dW, db, ws[:-256])
    restored = torch.full((N, d_in), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.sla_fp8_checkpoint_restore(ck[:-256], restored)
    torch.cuda.synchronize()
    assert torch.equal(kept, ck)
    assert bool((ck[-256:] == 0x5A).all()) and bool((ws[-256:] == 0x5A).all())
    (xc, xs), (wc, wsc) = po.e4m3_rows(x), po.e4m3_rows(W)
    xq, wq, g = xc * xs[:, None], wc * wsc[:, None], po.bf16_to_f64(dy)
    rx, rW, rb = po.fp8_linear_backward(x, W, g)
    # exact products, d_in fp32 sums, three roundings and the bf16 store
    ref = po.fp8_linear_train(x, W, b)
    assert (np.abs(f64(y) - ref) <= 2.0 ** -8 * np.abs(ref) + (d_in + 4) * 2.0 ** -24 * (np.abs(xq) @ np.abs(wq).T + np.abs(po.bf16_to_f64(b)))).all()
    want = torch.from_numpy((xc * xs[:, None]).astype(np.float32)).to(torch.bfloat16)
    assert (np.abs(f64(restored) - xq) <= 2.0 ** -8 * np.abs(xq) * (1 + 2.0 ** -15)).all() and (f64(restored) == f64(want)).mean() > 0.9999
    check(f64(dx), rx, np.abs(g) @ np.abs(wq), d_out, "dx")
    check(f64(dW), rW, np.abs(g).T @ np.abs(xq), N, "dW")
    assert (np.abs(f64(db) - rb) <= 2.0 ** -8 * np.abs(rb) + (N + 20) * 2.0 ** -24 * np.abs(g).sum(0)).all()
    # each alone, twice: dx the same bits, dW and db (another split of their sums) within the same bounds and the same bits both times
    first = {}
    for name in ("dx", "dW", "both", "dW", "both"):
        one = {"dx": dict(dx=torch.empty_like(dx)), "dW": dict(dW=torch.empty_like(dW)), "both": dict(dW=torch.empty_like(dW), db=torch.empty_like(db))}[name]
        B.sla_fp8_linear_grad(dyd, ck[:-256], Wd, workspace=ws[:-256], **one)
        torch.cuda.synchronize()
        for k, t in one.items():
            assert torch.equal(t.view(torch.int16), first.setdefault(k, dx if k == "dx" else t).view(torch.int16)), (name, k)
    check(f64(first["dW"]), rW, np.abs(g).T @ np.abs(xq), N, "dW alone")
    assert (np.abs(f64(first["db"]) - rb) <= 2.0 ** -8 * np.abs(rb) + (N + 20) * 2.0 ** -24 * np.abs(g).sum(0)).all()


def test_no_tokens_give_gradients_of_zero():
    dW, db = torch.full((72, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((72,), 3.0, dtype=torch.bfloat16, device="cuda")
    e = torch.empty((0, 72), dtype=torch.bfloat16, device="cuda")
    B.sla_fp8_linear_grad(e, torch.empty(256, dtype=torch.uint8, device="cuda"), torch.zeros((72, 128), dtype=torch.bfloat16, device="cuda"), dW=dW, db=db)
    torch.cuda.synchronize()
    assert bool((dW == 0).all()) and bool((db == 0).all())


def test_rows_of_zeros_and_a_gradient_of_infinity():
    x, W, b, dy = layer(70, 128, 40)
    x[5] = 0
    g = po.bf16_to_f64(dy)
    X, Wd, dyd = map(G.dev_bf16, (x, W, dy))
    ck, ws, y, dx, dW, db = buffers(70, 128, 40)
    B.sla_fp8_linear_save(X, Wd, None, y, ck)
    dyd[3, 7] = float("inf")
    B.sla_fp8_linear_grad(dyd, ck, Wd, dx, dW, db)
    torch.cuda.synchronize()
    rx, rW, rb = po.fp8_linear_backward(x, W, g)
    (xc, xs), (wc, wsc) = po.e4m3_rows(x), po.e4m3_rows(W)
    rows, outs = [i for i in range(70) if i != 3], [o for o in range(40) if o != 7]
    check(f64(dx)[rows], rx[rows], (np.abs(g) @ np.abs(wc * wsc[:, None]))[rows], 40, "dx")
    check(f64(dW)[outs], rW[outs], (np.abs(g).T @ np.abs(xc * xs[:, None]))[outs], 70, "dW")
    assert not np.isfinite(f64(dx)[3]).any() and not np.isfinite(f64(dW)[7]).all() and np.isinf(f64(db)[7]) and np.isfinite(f64(db)[outs]).all()


def test_gradients_are_those_of_the_quantised_product():
    """The difference quotient of the layer's own forward in dy's direction: y is linear in x_q, so <dy, y(x_q)> = <dx, x_q>."""
    x, W, b, dy = layer(130, 256, 64, 7)
    X, Wd, dyd = map(G.dev_bf16, (x, W, dy))
    ck, ws, y, dx, dW, db = buffers(130, 256, 64)
    B.sla_fp8_linear_save(X, Wd, None, y, ck)
    B.sla_fp8_linear_grad(dyd, ck, Wd, dx, dW)
    xq = B.sla_fp8_checkpoint_restore(ck, torch.empty_like(X))
    torch.cuda.synchronize()
    loss, size = float((f64(y) * f64(dyd)).sum()), float(np.abs(f64(y) * f64(dyd)).sum())
    (wc, wsc) = po.e4m3_rows(W)
    # y, dx, dW and x_q carry one or two bf16 roundings of random sign each: far below 1 % of the sum of magnitudes
    assert abs(float((f64(dx) * f64(xq)).sum()) - loss) < 0.01 * size
    assert abs(float((f64(dW) * (wc * wsc[:, None])).sum()) - loss) < 0.01 * size


def test_replays_from_a_graph():
    x, W, b, dy = layer(500, 256, 520)
    X, Wd, bd, dyd = map(G.dev_bf16, (x, W, b, dy))
    ck, ws, y, dx, dW, db = buffers(500, 256, 520)

    def work():
        B.sla_fp8_linear_save(X, Wd, bd, y, ck, ws)
        B.sla_fp8_linear_grad(dyd, ck, Wd, dx, dW, db, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(3):
        X.mul_(1.5), dyd.add_(0.01)
        work()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dW, db)]
        for t in (y, dx, dW, db, ck):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.int16), c.view(torch.int16)) for a, c in zip(want, (y, dx, dW, db))), k


def test_tensors_of_another_shape_type_or_place_are_refused():
    ck, ws, y, dx, dW, db = buffers(5, 128, 8)
    W, x = dW.clone(), dx.clone()
    for name, kw in [("dx", dict(dx=dx[:4])), ("db", dict(dW=dW, db=db[:4])), ("dW", dict(dW=dW.cpu())), ("workspace", dict(workspace=ws.float()))]:
        with pytest.raises(ValueError, match=name):
            B.sla_fp8_linear_grad(y, ck, W, **kw)
    with pytest.raises(ValueError, match="y: "):
        B.sla_fp8_linear_save(x, W, None, y.t(), ck)
    with pytest.raises(B.SlaError, match="checkpoint has"):
        B.sla_fp8_linear_grad(y, ck[:256], W, dW=dW)


def test_codes_are_pytorch_s():
    """amax / 448.0 written in PyTorch on the GPU, the division and the cast: the numbers that the checkpoint holds, bit for bit."""
    x = torch.from_numpy(np.random.default_rng(3).standard_normal((700, 256)).astype(np.float32)).cuda().to(torch.bfloat16)
    x[:128, 0] = torch.arange(128, 256, device="cuda").to(torch.bfloat16)                   # every significand as a row's maximum
    W = torch.zeros((8, 256), dtype=torch.bfloat16, device="cuda")
    ck = torch.empty(B.sla_fp8_checkpoint_bytes(700, 256), dtype=torch.uint8, device="cuda")
    B.sla_fp8_linear_save(x, W, None, torch.empty((700, 8), dtype=torch.bfloat16, device="cuda"), ck)
    xq = B.sla_fp8_checkpoint_restore(ck, torch.empty_like(x))
    scale = x.float().abs().amax(1, keepdim=True).clamp(min=1e-8) / 448.0
    want = (x.float() / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() * scale
    assert torch.equal(xq, want.to(torch.bfloat16))


@pytest.mark.parametrize("N,d_in,d_out", [(8213, 1152, 3208), (33001, 256, 4104)])
def test_large_tiles(N, d_in, d_out):
    """Sizes of the largest tiles, with ends inside a tile and inside a step on all three axes; fp64 products on the device."""
    x, W, b, dy = layer(N, d_in, d_out, 3)
    X, Wd, bd, dyd = map(G.dev_bf16, (x, W, b, dy))
    ck, ws, y, dx, dW, db = buffers(N, d_in, d_out)
    B.sla_fp8_linear_save(X, Wd, bd, y, ck[:-256], ws[:-256])
    B.sla_fp8_linear_grad(dyd, ck[:-256], Wd, dx, dW, db, ws[:-256])
    (xc, xs), (wc, wsc) = po.e4m3_rows(x), po.e4m3_rows(W)
    xq, wq = (torch.from_numpy(c * s[:, None]).cuda() for c, s in ((xc, xs), (wc, wsc)))
    g = dyd.double()
    for got, a, q, K, what in ((dx, g, wq, d_out, "dx"), (dW, g.T, xq, N, "dW")):
        ref, mag = a @ q, a.abs() @ q.abs()
        d = (got.double() - ref).abs()
        assert bool((d <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + (K + 20) * 2.0 ** -24) * mag).all()), (what, float(d.max()))
        assert float(torch.linalg.norm(got.double() - ref)) <= 3.2e-3 * float(torch.linalg.norm(ref)), what
    ref, mag = g.sum(0), g.abs().sum(0)
    assert bool(((db.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (N + 20) * 2.0 ** -24 * mag).all())
    ref = xq @ wq.T + bd.double()
    mag = xq.abs() @ wq.abs().T + bd.double().abs()
    assert bool(((y.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (d_in + 4) * 2.0 ** -24 * mag).all())
    assert bool((ck[-256:] == 0x5A).all()) and bool((ws[-256:] == 0x5A).all())
