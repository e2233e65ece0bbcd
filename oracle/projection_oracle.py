"""fp64 references of the operators around the attention: norm and rotation of heads with their gradients, the gradients of
the FP8 layer, the microscaled 4-bit format and its linear layer.

TEST INFRASTRUCTURE ONLY, numpy throughout: it never imports the GPU package and the GPU package never imports it.
"""
from __future__ import annotations

import numpy as np

from . import sla_oracle


def bf16_to_f64(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ---- norm and rotation of heads: rows x [B,N,H,64] of one tensor
def _angles(pos, axes, base, pairing):
    """(members i, members p, angle [1 or B, N, 32]) of the 32 pairs of channels; pos [N,axes] or [1 or B,N,axes]."""
    pos = np.asarray(pos, np.float64).reshape(-1, np.shape(pos)[-2], axes)
    S = 64 // axes
    first, second, ang = [], [], []
    for ax in range(axes):
        for j in range(S // 2):
            first.append(ax * S + (j if pairing == "halves" else 2 * j))
            second.append(ax * S + (j + S // 2 if pairing == "halves" else 2 * j + 1))
            ang.append(pos[..., ax] * base ** (-2.0 * j / S))
    return first, second, np.stack(ang, -1)


def _turn(t, axes, base, pairing, pos, back=False):
    if axes == 0:
        return t
    i, p, a = _angles(pos, axes, base, pairing)
    c, s = np.cos(a)[:, :, None, :], np.sin(a)[:, :, None, :] * (-1.0 if back else 1.0)
    out = t.copy()
    out[..., i] = t[..., i] * c - t[..., p] * s
    out[..., p] = t[..., p] * c + t[..., i] * s
    return out


def _unit(x, norm, eps):
    """u and r of the rows."""
    if norm == "none":
        return x, None
    d = x - x.mean(-1, keepdims=True) if norm == "layer" else x
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return d * r, r


def heads_forward(x, norm, w, b, eps, axes, pairing, base, pos):
    """w, b: None, [64] or [H,64]."""
    n, _ = _unit(x, norm, eps)
    n = n if w is None else n * w
    n = n if b is None else n + b
    return _turn(n, axes, base, pairing, pos)


def heads_backward(x, norm, w, eps, axes, pairing, base, pos, dy, per_head=False):
    """(dx, dw, db); dw and db are None without a norm."""
    d = _turn(dy, axes, base, pairing, pos, back=True)
    u, r = _unit(x, norm, eps)
    if r is None:
        return d, None, None
    over = (0, 1) if per_head else (0, 1, 2)
    g = d if w is None else d * w
    inner = g - (g * u).mean(-1, keepdims=True) * u
    if norm == "layer":
        inner = inner - g.mean(-1, keepdims=True)
    return r * inner, (d * u).sum(over), d.sum(over)


# ---- the FP8 layer's gradients
def e4m3_rows(bits):
    """(values, scales) of bf16 rows as the layer's training form quantises them: E4M3 numbers of fp32 quotients, one fp32 scale per
    row, max(amax, 1e-8) times the fp32 number 1/448."""
    x = (np.ascontiguousarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)
    scales = np.maximum(np.abs(x).max(-1), np.float32(1e-8)) * (np.float32(1) / np.float32(448))
    assert scales.dtype == np.float32
    codes = sla_oracle._e4m3_cast(np.clip(x / scales[:, None], np.float32(-448), np.float32(448)))
    return np.where(codes & 0x80, -1.0, 1.0) * sla_oracle._e4m3_grid()[(codes & 0x7F).astype(np.int64)], scales.astype(np.float64)


def fp8_linear_train(x_bits, W_bits, bias_bits):
    """y of the training form in exact products."""
    (xc, xs), (wc, ws) = e4m3_rows(x_bits), e4m3_rows(W_bits)
    return (xc * xs[:, None]) @ (wc * ws[:, None]).T + bf16_to_f64(bias_bits)


def fp8_linear_backward(x_bits, W_bits, dy):
    """(dx, dW, db), straight through both quantisers; dy float64 [N, d_out]."""
    (xc, xs), (wc, ws) = e4m3_rows(x_bits), e4m3_rows(W_bits)
    return dy @ (wc * ws[:, None]), dy.T @ (xc * xs[:, None]), dy.sum(0)


# ---- microscaled 4-bit numbers: by search through the sixteen numbers, ties to the even code
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mxfp4_quantise(bits):
    """(codes [rows, cols] 0 .. 15, scales [rows, cols/32]) of bf16 bit patterns [rows, cols]."""
    bits = np.asarray(bits, np.uint16)
    x = bf16_to_f64(bits).reshape(bits.shape[0], -1, 32)
    bad = ~np.isfinite(x).all(-1)
    mag = np.where(bad[..., None], 0.0, np.abs(x))
    s = np.maximum(np.where(mag.max(-1) > 0, np.frexp(mag.max(-1))[1] - 1, -200) + 125, 0)
    v = mag * np.ldexp(1.0, 127 - s)[..., None]
    d = np.abs(np.minimum(v, 6.0)[..., None] - E2M1)
    best = d.min(-1, keepdims=True)
    code = np.where(d == best, np.arange(8) + 8 * (np.arange(8) % 2), 99).min(-1) % 8        # of two at the same distance the even one
    code = code + 8 * (bits.reshape(x.shape) >> 15)
    code[bad] = 0
    return code.reshape(bits.shape), np.where(bad, 255, s)


def mxfp4_values(codes, scales):
    v = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    p = np.where(scales == 255, np.nan, np.ldexp(1.0, np.where(scales == 255, 0, scales) - 127))
    return v * np.repeat(p, 32, 1)


def mxfp4_pack(codes):
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)
