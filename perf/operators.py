"""Performance cases of the operators around the attention: what lies between a qkv projection and the attention, the
training step of the FP8 layer from an 8-bit copy of its input, and the linear layer in microscaled 4-bit numbers.

A case is a plain dict.  `kind` says what one pass is:
  heads   norm of every head's queries and keys, position rotation, and the layout (and, for "e4m3", the data type with its
          block scales) in which the attention takes Q, K and V; for "train" also the gradients of all of it
  ckpt    the FP8 fake-quantised linear layer that keeps its input in 8 bits, and its gradients from those 8 bits
  mx      the linear layer whose weights are kept as 4-bit floating point numbers with a power of two per 32 of them
  mxq     a matrix to that format and back
With `own` false, `run` computes the operators in elementary torch operations; with `own` true through the package.
"""
import math

import torch

own = False

DEV = "cuda:0"
FRAME = 1374          # tokens of a frame in the benchmark configurations: 1369 patches + 5 special tokens


def _heads(mode, Bn, N, H, norm="layer", per_head=False, axes=2, pairing="halves", base=100.0, source="fused", layout="bnhd", bq=64,
           v=True, own_pos=False):
    return dict(kind="heads", mode=mode, B=Bn, N=N, H=H, norm=norm, per_head=per_head, axes=axes, pairing=pairing, base=base,
                source=source, layout=layout, bq=bq, v=v, own_pos=own_pos)


def _ckpt(N, d_in, d_out, bias=True):
    return dict(kind="ckpt", N=N, d_in=d_in, d_out=d_out, bias=bias)


def _mx(N, d_in, d_out, bias=True):
    return dict(kind="mx", N=N, d_in=d_in, d_out=d_out, bias=bias)


def listed():
    return [
        # one new token of each of 32 sequences, every one at a far position of its own: the smallest call, latency alone
        dict(_heads("bf16", 32, 1, 16, norm="rms", axes=1, pairing="adjacent", base=1e6, own_pos=True), name="heads_token32"),
        # frame attention on eight frames: a (row, column) position for every patch, the same in all frames
        dict(_heads("bf16", 8, FRAME, 16, layout="bhnd"), name="heads_frames8"),
        # global attention over 32 frames on the E4M3 path: 128-row query blocks with their scales
        dict(_heads("e4m3", 1, 32 * FRAME, 16, bq=128), name="heads_global32_e4m3"),
        # training on two ragged sequences, weights for each head, heads interleaved as [head][q k v]
        dict(_heads("train", 2, 5 * FRAME + 37, 12, per_head=True, source="per_head", own_pos=True), name="heads_train_ragged"),
        # a small layer on a short odd number of tokens: launches and latency
        dict(_ckpt(197, 384, 1152), name="ckpt_small"),
        # the output projection of a global layer over eight frames
        dict(_ckpt(8 * FRAME, 1024, 1024), name="ckpt_out8"),
        # the first layer of the feed-forward block over 32 frames, the largest call
        dict(_ckpt(32 * FRAME, 1024, 4096), name="ckpt_ff32"),
        # one token through a wide layer: the weights are read once, nothing else counts
        dict(_mx(1, 4096, 4096), name="mx_token"),
        # a few tokens, an odd number of them
        dict(_mx(9, 2048, 8200, bias=False), name="mx_few"),
        # one frame through the feed-forward block's first layer
        dict(_mx(FRAME, 1024, 4096), name="mx_frame"),
        # 32 frames through its second layer
        dict(_mx(32 * FRAME, 4096, 1024), name="mx_ff32"),
        # a large activation matrix to 4 bits and back
        dict(kind="mxq", rows=32 * FRAME - 5, cols=1024, name="mx_quantise"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "heads", "heads", "ckpt", "ckpt", "mx", "mx", "mx", "mxq"])
    if kind == "heads":
        mode = rng.choice(["bf16", "e4m3", "train"])
        H = rng.choice([1, 2, 3, 6, 8, 12, 16, 16])
        Bn = rng.choice([1, 1, 2, _log_int(rng, 1, 64)])
        N = min(_log_int(rng, 1, 44000), 44000 * 16 // (Bn * H))
        axes = rng.choice([0, 1, 2, 2])
        return _heads(mode, Bn, N, H, norm=rng.choice(["layer", "layer", "rms", "none"]), per_head=rng.random() < 0.3, axes=axes,
                      pairing=rng.choice(["halves", "halves", "adjacent"]), base=rng.choice([100.0, 1e4, 1e6]),
                      source=rng.choice(["fused", "fused", "per_head", "split", "head_major"]), layout=rng.choice(["bhnd", "bnhd"]),
                      bq=rng.choice([64, 128]), v=rng.random() < 0.8, own_pos=rng.random() < 0.4)
    if kind == "mxq":
        cols = 32 * rng.randint(1, 160)
        return dict(kind="mxq", rows=min(_log_int(rng, 1, 44000), 44000 * 1024 // cols), cols=cols)
    d_in, d_out = 128 * _log_int(rng, 1, 32), 8 * _log_int(rng, 8, 1024)
    N = min(_log_int(rng, 1, 44000), 43968 * 1024 * 4096 // (d_in * d_out))
    if kind == "mx" and rng.random() < 0.4:
        N = _log_int(rng, 1, 64)
    return (_ckpt if kind == "ckpt" else _mx)(N, d_in, d_out, rng.random() < 0.7)


def _blocks(n, blk):
    return -(-n // blk)


# ------------------------------------------------------------------------------------------------------------ inputs
def _activations(gen, *shape):
    """bf16 activations as layers meet them: a level for each token, channels of different size, a few of them large."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn((*shape[:-1], 1), generator=gen, device=DEV))
    size = torch.exp(0.4 * torch.randn(shape[-1], generator=gen, device=DEV))
    size = torch.where(torch.rand(shape[-1], generator=gen, device=DEV) < 0.01, 8.0 * size, size)
    return x.mul_(size).add_(0.2 * torch.randn(shape[-1], generator=gen, device=DEV)).to(torch.bfloat16)


def _three(source, Bn, N, H):
    """An empty buffer for the q, k, v of a projection's output, and the three as [B,N,H,64] views of it."""
    if source == "fused":                 # [q|k|v][head][64] along a token's row
        t = torch.empty((Bn, N, 3, H, 64), dtype=torch.bfloat16, device=DEV)
        return t, [t[:, :, i] for i in range(3)]
    if source == "per_head":              # [head][q|k|v][64] along a token's row
        t = torch.empty((Bn, N, H, 3, 64), dtype=torch.bfloat16, device=DEV)
        return t, [t[:, :, :, i] for i in range(3)]
    if source == "head_major":            # three tensors [B,H,N,64]
        t = torch.empty((3, Bn, H, N, 64), dtype=torch.bfloat16, device=DEV)
        return t, [t[i].transpose(1, 2) for i in range(3)]
    t = torch.empty((3, Bn, N, H, 64), dtype=torch.bfloat16, device=DEV)      # three tensors [B,N,H,64]
    return t, [t[i] for i in range(3)]


def _positions(case, gen):
    """int32 [1 or B, N, axes]: (row, column) of the patches of frames 37 patches wide, special tokens at 0; on one axis the
    place in the sequence, for single tokens far into it."""
    Bn, N, axes = case["B"], case["N"], case["axes"]
    if axes == 0:
        return None
    t = torch.arange(N, device=DEV)
    if axes == 1:
        p = t[None, :, None].repeat(Bn if case["own_pos"] else 1, 1, 1)
        if case["own_pos"]:
            p = p + torch.randint(0, 200000, (Bn, 1, 1), generator=gen, device=DEV)
    else:
        i = t % FRAME - 5
        p = torch.stack([torch.where(i < 0, 0, i // 37 + 1), torch.where(i < 0, 0, i % 37 + 1)], -1)[None]
        if case["own_pos"]:
            p = p + torch.randint(0, 16, (Bn, 1, 2), generator=gen, device=DEV)
    return p.to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    st = {"case": case}
    bf = dict(dtype=torch.bfloat16, device=DEV)
    if case["kind"] == "heads":
        Bn, N, H, mode = case["B"], case["N"], case["H"], case["mode"]
        buf, st["qkv"] = _three(case["source"], Bn, N, H)
        for t in st["qkv"]:
            t.copy_(_activations(gen, Bn, N, H, 64))
        st["buf"] = buf
        shape = (H, 64) if case["per_head"] else (64,)
        par = lambda at, by: at + by * torch.randn(shape, generator=gen, device=DEV)      # fp32, as norms keep their parameters
        st["w"] = [par(1.0, 0.2), par(1.0, 0.2)] if case["norm"] != "none" else [None, None]
        st["b"] = [par(0.0, 0.1), par(0.0, 0.1)] if case["norm"] == "layer" else [None, None]
        st["pos"] = _positions(case, gen)
        out = (Bn, N, H, 64) if case["layout"] == "bnhd" else (Bn, H, N, 64)
        three = 3 if case["v"] else 2
        if mode == "e4m3":
            st["out"] = [torch.empty(out, dtype=torch.uint8, device=DEV) for _ in range(three)]
            st["scales"] = [torch.empty((Bn, H, _blocks(N, blk)), device=DEV) for blk in (case["bq"], 64, 64)[:three]]
        else:
            st["out"] = [torch.empty(out, **bf) for _ in range(three)]
        if mode == "train":
            st["grads"] = [_activations(gen, *out).mul_(0.01) for _ in range(three)]
            st["dbuf"], st["dqkv"] = _three(case["source"], Bn, N, H)
            st["dw"] = [torch.empty_like(w) if w is not None else None for w in st["w"]]
            st["db"] = [torch.empty_like(b) if b is not None else None for b in st["b"]]
        if own:                           # the plan of the call: sizes, strides and options in one struct
            from paper_2605_11354_amd import binding as B
            st["p"] = B.make_heads_params(st["qkv"][0], norm=case["norm"], norm_per_head=case["per_head"], axes=case["axes"],
                                          pairing=case["pairing"], base=case["base"], pos_per_item=case["own_pos"], layout=case["layout"])
        return st
    if case["kind"] == "mxq":
        st["x"] = _activations(gen, case["rows"], case["cols"])
        st["codes"] = torch.empty((case["rows"], case["cols"] // 2), dtype=torch.uint8, device=DEV)
        st["scales"] = torch.empty((case["rows"], case["cols"] // 32), dtype=torch.uint8, device=DEV)
        st["y"] = torch.empty((case["rows"], case["cols"]), **bf)
        return st
    N, d_in, d_out = case["N"], case["d_in"], case["d_out"]
    st["x"] = _activations(gen, N, d_in)
    W = (torch.randn((d_out, d_in), generator=gen, device=DEV) * torch.exp(0.3 * torch.randn((d_out, 1), generator=gen, device=DEV)) / d_in ** 0.5).to(torch.bfloat16)
    st["bias"] = torch.randn((d_out,), generator=gen, device=DEV).to(torch.bfloat16) if case["bias"] else None
    st["y"] = torch.empty((N, d_out), **bf)
    if case["kind"] == "mx":              # the weights as a program keeps them: codes and scales
        st["Wc"], st["Ws"] = _pack_mx(*_to_mx(W))
        st["ws"] = torch.empty(N * d_in + 4096, dtype=torch.uint8, device=DEV)
        return st
    st["W"], st["dy"] = W, _activations(gen, N, d_out).mul_(0.01)
    st["dx"], st["dW"] = torch.empty((N, d_in), **bf), torch.empty((d_out, d_in), **bf)
    st["db"] = torch.empty((d_out,), **bf) if case["bias"] else None
    if own:                               # a training program keeps one of each: the 8-bit copy for a layer, the scratch for all
        from paper_2605_11354_amd import binding as B
        st["ckpt"] = torch.empty(B.sla_fp8_checkpoint_bytes(N, d_in), dtype=torch.uint8, device=DEV)
        st["ws"] = torch.empty(B.sla_fp8_linear_grad_workspace_bytes(N, d_in, d_out), dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------------------------------------------------------------- the plain forms
def _cos_sin(case, pos):
    """fp32 [1 or B, N, 1, axes, S/2] each; the angle itself in 64 bits, since positions reach hundreds of thousands."""
    S = 64 // case["axes"]
    freq = case["base"] ** (-2.0 * torch.arange(S // 2, dtype=torch.float64, device=DEV) / S)
    ang = pos.double()[:, :, None, :, None] * freq
    return torch.cos(ang).float(), torch.sin(ang).float()


def _pairs(case, t):
    """The two members of every rotated pair of t [B,N,H,64]: [B,N,H,axes,S/2] each."""
    t = t.reshape(*t.shape[:3], case["axes"], 64 // case["axes"])
    half = t.shape[-1] // 2
    return (t[..., :half], t[..., half:]) if case["pairing"] == "halves" else (t[..., 0::2], t[..., 1::2])


def _join(case, a, b, shape):
    return (torch.cat([a, b], -1) if case["pairing"] == "halves" else torch.stack([a, b], -1)).reshape(shape)


def _norm(case, x):
    """(normalised values, factor of the deviation) of the rows of x, before the weights."""
    if case["norm"] == "none":
        return x, None
    if case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5)
    return x * r, r


def _heads_one(case, x, w, b, cs):
    n, _ = _norm(case, x.float())
    if w is not None:
        n = n * w
    if b is not None:
        n = n + b
    if cs is not None:
        a, c = _pairs(case, n)
        n = _join(case, a * cs[0] - c * cs[1], c * cs[0] + a * cs[1], n.shape)
    return n


def _heads_one_grad(case, x, w, dn, cs):
    """Gradients of _heads_one's input, weight and bias from that of its result, dn [B,N,H,64] fp32."""
    if cs is not None:
        a, c = _pairs(case, dn)
        dn = _join(case, a * cs[0] + c * cs[1], c * cs[0] - a * cs[1], dn.shape)
    xh, r = _norm(case, x.float())
    if r is None:
        return dn, None, None
    over = (0, 1) if case["per_head"] else (0, 1, 2)
    dw, db = (dn * xh).sum(over), dn.sum(over)
    g = dn * w
    g = g - xh * (g * xh).mean(-1, keepdim=True) - (g.mean(-1, keepdim=True) if case["norm"] == "layer" else 0.0)
    return g * r, dw, db


def _blockwise(y, blk):
    """E4M3 codes of y [B,N,H,64] and the scales [B,H,blocks] of blocks of `blk` tokens of a head."""
    Bn, N, H, _ = y.shape
    full = torch.zeros((Bn, _blocks(N, blk) * blk, H, 64), dtype=y.dtype, device=DEV)
    full[:, :N] = y
    full = full.reshape(Bn, -1, blk, H, 64)
    scale = full.abs().amax((2, 4)).clamp(min=1e-8) / 448.0
    codes = (full / scale[:, :, None, :, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return codes.reshape(Bn, -1, H, 64)[:, :N], scale.transpose(1, 2).contiguous()


def _heads_plain(st):
    case = st["case"]
    cs = _cos_sin(case, st["pos"]) if case["axes"] else None
    place = (lambda t: t.contiguous()) if case["layout"] == "bnhd" else (lambda t: t.transpose(1, 2).contiguous())
    q, k, v = st["qkv"]
    ys = [_heads_one(case, x, w, b, cs) for x, w, b in zip((q, k), st["w"], st["b"])] + ([v.float()] if case["v"] else [])
    if case["mode"] == "e4m3":
        both = [_blockwise(y, blk) for y, blk in zip(ys, (case["bq"], 64, 64))]
        return {"codes": [place(c) for c, _ in both], "scales": [s for _, s in both]}
    out = {"out": [place(y.to(torch.bfloat16)) for y in ys]}
    if case["mode"] == "train":
        back = [g if case["layout"] == "bnhd" else g.transpose(1, 2) for g in st["grads"]]
        got = [_heads_one_grad(case, x, w, g.float(), cs) for x, w, g in zip((q, k), st["w"], back)]
        out["dqkv"] = [g[0].to(torch.bfloat16) for g in got] + ([back[2].contiguous()] if case["v"] else [])
        out["dw"] = [g[1] if w is not None else None for g, w in zip(got, st["w"])]
        out["db"] = [g[2] if b is not None else None for g, b in zip(got, st["b"])]
    return out


def _to_e4m3_rows(x):
    """x as E4M3 numbers times a scale for each row: (values, scales), both fp32."""
    x = x.float()
    scale = x.abs().amax(1, keepdim=True).clamp(min=1e-8) / 448.0
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float(), scale


def _ckpt_plain(st):
    xc, xs = _to_e4m3_rows(st["x"])
    wc, ws = _to_e4m3_rows(st["W"])
    xq, wq, dy = xc * xs, wc * ws, st["dy"].float()
    y = xq @ wq.t()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    out = {"y": y.to(torch.bfloat16), "dx": (dy @ wq).to(torch.bfloat16), "dW": (dy.t() @ xq).to(torch.bfloat16)}
    if st["bias"] is not None:
        out["db"] = dy.sum(0).to(torch.bfloat16)
    return out


def _to_mx(x):
    """x [rows, cols] as 4-bit floating point numbers times a power of two for every 32 of a row: the numbers, fp32
    [rows, cols/32, 32], and the exponents of the powers plus 127, int32 [rows, cols/32]."""
    x = x.float().reshape(x.shape[0], -1, 32)
    e = ((x.abs().amax(-1).view(torch.int32) >> 23) - 2).clamp(min=0)           # largest number of the format: 1.5 * 2^2
    v = x * ((254 - e) << 23).view(torch.float32)[..., None]
    m = v.abs()
    m = torch.where(m < 2.0, torch.round(2.0 * m) * 0.5, torch.where(m < 4.0, torch.round(m), torch.round(0.5 * m) * 2.0)).clamp(max=6.0)
    return torch.copysign(m, v), e


def _pack_mx(v, e):
    """Codes (sign, two bits of exponent, one of mantissa; the even element in the low half of a byte) and scales as bytes."""
    m = v.abs()
    code = torch.where(m < 2.0, 2.0 * m, torch.where(m < 4.0, m + 2.0, 0.5 * m + 4.0)).to(torch.int32) + 8 * torch.signbit(v)
    code = code.reshape(code.shape[0], -1)
    return (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8), e.to(torch.uint8)


def _power(e):
    """2^(e - 127) for int32 e in 0 .. 254."""
    return torch.where(e > 0, (e << 23).view(torch.float32), 2.0 ** -127)


def _from_mx(codes, scales):
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    grid = torch.cat([grid, -grid])
    v = torch.stack([grid[(codes & 15).int()], grid[(codes >> 4).int()]], -1).reshape(codes.shape[0], -1, 32)
    return (v * _power(scales.int())[..., None]).reshape(codes.shape[0], -1)


def _mx_plain(st):
    v, e = _to_mx(st["x"])
    xq = (v * _power(e)[..., None]).reshape(st["x"].shape)
    if st["case"]["kind"] == "mxq":
        return {"y": xq.to(torch.bfloat16)}
    y = xq @ _from_mx(st["Wc"], st["Ws"]).t()
    if st["bias"] is not None:
        y = y + st["bias"].float()
    return {"y": y.to(torch.bfloat16)}


# -------------------------------------------------------------------------------------------------------------- pass
def _own(st):
    from paper_2605_11354_amd import binding as B
    case = st["case"]
    if case["kind"] == "heads":
        q, k, v = st["qkv"] if case["v"] else (*st["qkv"][:2], None)
        Q, K, V = st["out"] if case["v"] else (*st["out"], None)
        par = dict(pos=st["pos"], q_weight=st["w"][0], k_weight=st["w"][1])
        bias = dict(q_bias=st["b"][0], k_bias=st["b"][1])
        if case["mode"] == "e4m3":
            s = st["scales"] if case["v"] else (*st["scales"], None)
            B.sla_qk_norm_rope_e4m3(st["p"], q, k, v, case["bq"], Q, K, V, *s, **par, **bias)
            return {"codes": [t.view(torch.float8_e4m3fn) for t in st["out"]], "scales": st["scales"]}
        B.sla_qk_norm_rope(st["p"], q, k, v, Q, K, V, **par, **bias)
        out = {"out": st["out"]}
        if case["mode"] == "train":
            gQ, gK, gV = st["grads"] if case["v"] else (*st["grads"], None)
            dq, dk, dv = st["dqkv"] if case["v"] else (*st["dqkv"][:2], None)
            B.sla_qk_norm_rope_grad(st["p"], q, k, gQ, gK, gV, dq, dk, dv, **par, dq_weight=st["dw"][0], dq_bias=st["db"][0],
                                    dk_weight=st["dw"][1], dk_bias=st["db"][1])
            out |= {"dqkv": st["dqkv"] if case["v"] else st["dqkv"][:2], "dw": st["dw"], "db": st["db"]}
        return out
    if case["kind"] == "ckpt":
        B.sla_fp8_linear_save(st["x"], st["W"], st["bias"], st["y"], st["ckpt"], st["ws"])
        B.sla_fp8_linear_grad(st["dy"], st["ckpt"], st["W"], st["dx"], st["dW"], st["db"], st["ws"])
        return {k: st[k] for k in ("y", "dx", "dW", "db") if st[k] is not None}
    if case["kind"] == "mxq":
        B.sla_quantise_mxfp4(st["x"], st["codes"], st["scales"])
        return {"y": B.sla_dequantise_mxfp4(st["codes"], st["scales"], st["y"])}
    return {"y": B.sla_mxfp4_linear(st["x"], st["Wc"], st["Ws"], st["bias"], st["y"], st["ws"])}


def run(st):
    if own:
        return _own(st)
    return {"heads": _heads_plain, "ckpt": _ckpt_plain, "mx": _mx_plain, "mxq": _mx_plain}[st["case"]["kind"]](st)


# -------------------------------------------------------------------------------------------------------------- work
def work(case):
    if case["kind"] == "heads":
        rows, mode = case["B"] * case["N"] * case["H"], case["mode"]
        three = 3 if case["v"] else 2
        pos = 4 * case["N"] * case["axes"] * (case["B"] if case["own_pos"] else 1)
        per = {"bf16": 4 * three, "e4m3": 3 * three, "train": 4 * three + 4 * three}[mode]      # train: grads in, grads out too
        return {"bytes": rows * 64 * per + pos, "flops": 2.0 * rows * 64 * (24 if mode == "train" else 10)}
    if case["kind"] == "mxq":
        n = case["rows"] * case["cols"]
        return {"bytes": 4 * n + n / 2 + n / 32, "flops": 4.0 * n}
    N, d_in, d_out = case["N"], case["d_in"], case["d_out"]
    if case["kind"] == "mx":
        return {"bytes": 2 * N * (d_in + d_out) + d_out * d_in * 17 / 32 + (2 * d_out if case["bias"] else 0), "flops": 2.0 * N * d_in * d_out}
    return {"bytes": 4 * N * (d_in + d_out) + 4 * d_out * d_in + (4 * d_out if case["bias"] else 0), "flops": 6.0 * N * d_in * d_out}


# ------------------------------------------------------------------------------------------------- in 64 bits
def _exact_heads(st):
    """From the complex numbers that the pairs stand for, one tensor at a time."""
    case = st["case"]
    per = 32 // case["axes"] if case["axes"] else 0
    turn = None
    if case["axes"]:
        i = torch.arange(per, dtype=torch.float64, device=DEV)
        ang = st["pos"].double().unsqueeze(-1) / torch.pow(torch.tensor(case["base"], dtype=torch.float64, device=DEV), i / per)
        turn = torch.polar(torch.ones_like(ang), ang)[:, :, None]               # [1 or B, N, 1, axes, S/2]

    def complex_of(t):
        t = t.reshape(*t.shape[:-1], case["axes"], 2 * per)
        t = t.unflatten(-1, (2, per)).transpose(-1, -2) if case["pairing"] == "halves" else t.unflatten(-1, (per, 2))
        return torch.view_as_complex(t.contiguous())

    def real_of(z, shape):
        t = torch.view_as_real(z)
        return (t.transpose(-1, -2) if case["pairing"] == "halves" else t).reshape(shape)

    place = (lambda t: t) if case["layout"] == "bnhd" else (lambda t: t.transpose(1, 2))
    res = {"out": [], "codes": [], "scales": [], "dqkv": [], "dw": [], "db": []}
    for n, x in enumerate(st["qkv"][: 3 if case["v"] else 2]):
        x = x.double()
        w = st["w"][n].double() if n < 2 and st["w"][n] is not None else None
        b = st["b"][n].double() if n < 2 and st["b"][n] is not None else None
        u, r = x, None
        if n < 2 and case["norm"] != "none":
            m = x.mean(-1, keepdim=True) if case["norm"] == "layer" else 0.0
            r = ((x - m).square().mean(-1, keepdim=True) + 1e-5).rsqrt()
            u = (x - m) * r
        y = u if w is None else u * w if b is None else u * w + b
        if n < 2 and turn is not None:
            y = real_of(complex_of(y) * turn, y.shape)
        if case["mode"] == "e4m3":        # the values whose nearest 8-bit numbers are wanted, and the scales
            blk = case["bq"] if n == 0 else 64
            Bn, N, H, _ = y.shape
            top = torch.nn.functional.pad(y.abs().amax(-1), (0, 0, 0, -N % blk)).reshape(Bn, -1, blk, H).amax(2)
            s = (top.clamp(min=1e-8) / 448.0)
            res["scales"].append(s.transpose(1, 2))
            res["codes"].append(place(y / s.repeat_interleave(blk, 1)[:, :N, :, None]))
            continue
        res["out"].append(place(y))
        if case["mode"] != "train":
            continue
        g = st["grads"][n].double()
        g = g if case["layout"] == "bnhd" else g.transpose(1, 2)
        if n < 2 and turn is not None:
            g = real_of(complex_of(g) * turn.conj(), g.shape)
        if n < 2:
            over = (0, 1) if case["per_head"] else (0, 1, 2)
            res["dw"].append((g * u).sum(over) if w is not None else None)
            res["db"].append(g.sum(over) if b is not None else None)
            if w is not None:
                g = g * w
                along = (g * u).mean(-1, keepdim=True)
                g = r * (g - u * along - (g.mean(-1, keepdim=True) if case["norm"] == "layer" else 0.0))
        res["dqkv"].append(g)
    keys = {"bf16": ["out"], "e4m3": ["codes", "scales"], "train": ["out", "dqkv", "dw", "db"]}[case["mode"]]
    return {k: res[k] for k in keys}


def _two(e):
    """2^e in 64 bits, from the bits of the number."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_e4m3(x):
    """The layer's quantiser is defined in fp32 (scale and quotient); its numbers are rounded here from the bits of a quotient."""
    x = x.float()
    scale = torch.maximum(x.abs().max(1, keepdim=True).values, torch.tensor(1e-8, device=DEV)) / 448.0
    q = (x / scale).clamp(-448.0, 448.0).double()
    _, e = torch.frexp(q)
    step = _two((e - 4).clamp(min=-9))                                           # four significant bits, none below 2^-9
    return torch.round(q / step) * step * scale.double()


def _exact_mx(x):
    x = x.double().unflatten(1, (-1, 32))
    _, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    s = _two((e - 3).clamp(min=-127))
    q = x / s
    _, e = torch.frexp(q)
    step = _two((e - 2).clamp(min=-1))                                           # two significant bits, none below a half
    return ((torch.round(q / step) * step).clamp(-6.0, 6.0) * s).flatten(1)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "heads":
        return _exact_heads(st)
    xq = (_exact_e4m3 if case["kind"] == "ckpt" else _exact_mx)(st["x"])
    if case["kind"] == "mxq":
        return {"y": xq}
    bias = st["bias"].double() if st["bias"] is not None else 0.0
    if case["kind"] == "mx":
        nibble = torch.stack([st["Wc"] % 16, torch.div(st["Wc"], 16, rounding_mode="floor")], -1).flatten(1).double()
        m, ex = nibble % 2, torch.floor(nibble / 2) % 4
        size = torch.where(ex > 0, (1.0 + 0.5 * m) * _two(ex - 1.0), 0.5 * m)
        wq = torch.where(nibble >= 8, -size, size) * _two(st["Ws"].long() - 127).repeat_interleave(32, 1)
        return {"y": xq @ wq.t() + bias}
    wq, dy = _exact_e4m3(st["W"]), st["dy"].double()
    out = {"y": xq @ wq.t() + bias, "dx": dy @ wq, "dW": dy.t() @ xq}
    if st["bias"] is not None:
        out["db"] = dy.sum(0)
    return out
