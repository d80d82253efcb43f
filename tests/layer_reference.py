"""Plain forms in double of the layer operators, with the magnitudes their error bounds are stated in.

u(type) is half a unit in the last place, relative: 2^-24 fp32, 2^-11 fp16, 2^-8 bf16.  Every bound is
    u(out) |ref| + c * 2^-24 * mag + smallest step of the type
where mag is the sum of the absolute values of the terms and c counts the fp32 roundings a term goes through.
"""
import math

import numpy as np
import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
EPS32 = 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def assert_close(got, ref, mag, c, what, extra=0.0):
    """got: tensor; ref, mag: double arrays; c roundings of 2^-24 (plus `extra`, relative to mag)."""
    dtype, got = got.dtype, f64(got)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bound = U[dtype] * np.abs(ref) + (c * EPS32 + extra) * mag + TINY[dtype]
    bad = ~(np.abs(got - ref) <= bound)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} outside the bound; first at {i}: got {got[i]!r} "
                             f"want {ref[i]!r} (off {abs(got[i] - ref[i]):.3g}, bound {bound[i]:.3g})")


# ---------------------------------------------------------------------------------------------- linear

_erf = np.vectorize(math.erf, otypes=[float])


def act(y, kind):
    if kind == 1:
        return np.maximum(y, 0.0)
    if kind == 2:
        return 0.5 * y * (1.0 + _erf(y / math.sqrt(2.0)))
    if kind == 3:
        return 0.5 * y * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    if kind == 4:
        return y / (1.0 + np.exp(-y))
    return y


def linear(x, w, a_scale, a_offset, w_scale, w_offset, bias=None, kind=0, residual=None):
    """Codes and parameters as numpy arrays -> (ref, mag)."""
    a = np.asarray(a_scale, np.float64).reshape(-1, 1) * x + np.asarray(a_offset, np.float64).reshape(-1, 1)
    b = np.asarray(w_scale, np.float64).reshape(-1, 1) * w + np.asarray(w_offset, np.float64).reshape(-1, 1)
    K = x.shape[1]
    s, o = np.abs(np.asarray(a_scale, np.float64)).reshape(-1, 1), np.abs(np.asarray(a_offset, np.float64)).reshape(-1, 1)
    ws, wo = np.abs(np.asarray(w_scale, np.float64)).reshape(1, -1), np.abs(np.asarray(w_offset, np.float64)).reshape(1, -1)
    x64, w64 = x.astype(np.float64), w.astype(np.float64)
    # the four terms of the affine form, as the kernels add them up
    mag = s * ws * np.abs(x64 @ w64.T) + s * wo * np.abs(x64.sum(1, keepdims=True)) + o * ws * np.abs(w64.sum(1)) + K * o * wo
    y = a @ b.T
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    y = act(y, kind)
    if residual is not None:
        y, mag = y + residual, mag + np.abs(residual)
    return y, mag


# ---------------------------------------------------------------------------------------------- rotation

def rotary(x, positions, table, weight, eps, layout):
    """x [T, H, D], table [P, R] or None, all double -> (ref, mag)."""
    y = x.copy()
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * weight
    mag = np.abs(y)
    if table is None or table.shape[1] == 0:
        return y, mag
    R = table.shape[1]
    c, s = table[positions][:, None, :R // 2], table[positions][:, None, R // 2:]
    at = (slice(0, R // 2), slice(R // 2, R)) if layout == 0 else (slice(0, R, 2), slice(1, R, 2))
    a, b = y[..., at[0]], y[..., at[1]]
    out = y.copy()
    out[..., at[0]], out[..., at[1]] = a * c - b * s, b * c + a * s
    mag[..., at[0]], mag[..., at[1]] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return out, mag


# ---------------------------------------------------------------------------------------------- decay attention

def decay(q, k, v, log_decay, start, state, scale):
    """Token by token in double.  q [T, H, Dk], k [T, Hk, Dk], v [T, Hk, Dv]; state [B, H, Dk, Dv] or None.
    Returns out, mag_out, state, mag_state: the magnitudes are the recurrence on absolute values."""
    T, H, Dk = q.shape
    group = np.arange(H) // (H // k.shape[1])
    B, Dv = len(start) - 1, v.shape[2]
    keep = np.exp(log_decay.astype(np.float64))[:, None, None]
    out, mag = np.zeros((T, H, Dv)), np.zeros((T, H, Dv))
    ends, mags = np.zeros((B, H, Dk, Dv)), np.zeros((B, H, Dk, Dv))
    for b in range(B):
        S = np.zeros((H, Dk, Dv)) if state is None else state[b].astype(np.float64)
        A = np.abs(S)
        for t in range(start[b], start[b + 1]):
            kv = k[t][group][:, :, None] * v[t][group][:, None, :]
            S, A = keep * S + kv, keep * A + np.abs(kv)
            out[t] = scale * np.einsum("hi,hij->hj", q[t], S)
            mag[t] = abs(scale) * np.einsum("hi,hij->hj", np.abs(q[t]), A)
        ends[b], mags[b] = S, A
    return out, mag, ends, mags


def decay_roundings(log_decay, longest, Dk):
    """Roundings a term goes through: two per step it lives in the state (a step's factor shrinks what came before, so at most
    about two per 1 - l of them count), exp(log_decay)'s own error once per step, and the sum over Dk."""
    l = float(np.exp(np.max(log_decay)))
    steps = longest if l >= 1.0 else min(longest, 4.0 / (1.0 - l))
    return 4.0 * steps + Dk + 16.0
