"""The 8-bit cache written plainly, in 64 bits on the CPU (shared by the tests
of its writer, its reader and the attention over it)."""
from __future__ import annotations

import copy
import math

import numpy as np
import torch

from paper_2606_00024_amd import api

FORMATS = ["e4m3", "int8"]
DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}


def table(form: str) -> np.ndarray:
    """What each of the 256 codes stands for (fp64; NaN for e4m3's 0x7f, 0xff)."""
    if form == "int8":
        return np.array([c if c < 128 else c - 256 for c in range(256)], dtype=np.float64)
    out = []
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out.append(math.nan if (c & 127) == 127 else (-x if c >> 7 else x))
    return np.array(out)


def encode(x: np.ndarray, form: str) -> np.ndarray:
    """Codes nearest to x, ties to the even code; beyond the largest code, that
    code; NaN is NaN (e4m3) or 0 (int8)."""
    x = np.asarray(x, dtype=np.float64)
    if form == "int8":
        return np.nan_to_num(np.rint(np.clip(x, -127, 127)), nan=0.0).astype(np.int8).view(np.uint8)
    vals = table(form)[:127]                       # 0 .. 448, increasing, code = index
    a = np.clip(np.abs(np.nan_to_num(x, nan=0.0)), 0, 448.0)
    hi = np.clip(np.searchsorted(vals, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = vals[hi] - a, a - vals[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(a == vals[hi], hi, code).astype(np.uint8)
    code = code | (np.signbit(x).astype(np.uint8) << 7)
    return np.where(np.isnan(x), 0x7F, code & np.where(np.isnan(x), 0x7F, 0xFF)).astype(np.uint8)


def need(a: float, form: str) -> float:
    """Smallest 2^e, e >= -120, with a <= top * 2^e."""
    e = -120
    while math.ldexp(TOP[form], e) < a:
        e += 1
    return math.ldexp(1.0, e)


def append(codes, scale, rows, pages, positions, offsets, form):
    """codes uint8 [P][H][Ps][D], scale fp32 [P][H][runs], both changed in place;
    rows fp64 [n][H][D]; offsets B + 1 ints; everything numpy."""
    P, H, Ps, D = codes.shape
    run = Ps // scale.shape[2]
    vals, cap = table(form), pages.shape[1] * Ps
    for b, pos in enumerate(positions):
        first, end = offsets[b], offsets[b + 1]
        if pos < 0 or first == end:
            continue
        t = pos
        while t < pos + end - first and t < cap:
            stop = min((t // run + 1) * run, pos + end - first, cap)
            page, slot = pages[b, t // Ps], t % Ps
            if 0 <= page < P:
                old = t % run if t == pos else 0
                for h in range(H):
                    x = rows[first + t - pos: first + stop - pos, h]
                    mags = np.abs(x[np.isfinite(x)])
                    s = need(float(mags.max()) if mags.size else 0.0, form)
                    was = float(scale[page, h, slot // run])
                    if old:
                        s = max(s, was)
                        if s != was:
                            c = codes[page, h, slot - old: slot]
                            codes[page, h, slot - old: slot] = encode(vals[c] * (was / s), form)
                    scale[page, h, slot // run] = s
                    codes[page, h, slot: slot + stop - t] = encode(x / s, form)
            t = stop


def read(codes, scale, pages, positions, offsets, rows, form):
    """fp64 [rows][H][D]; NaN for rows of no token."""
    P, H, Ps, D = codes.shape
    run = Ps // scale.shape[2]
    out = np.full((rows, H, D), np.nan)
    vals = table(form)
    for b, pos in enumerate(positions):
        for r in range(offsets[b], offsets[b + 1]):
            t = pos + r - offsets[b]
            if pos < 0 or t >= pages.shape[1] * Ps or not 0 <= pages[b, t // Ps] < P:
                continue
            page, slot = pages[b, t // Ps], t % Ps
            out[r] = vals[codes[page, :, slot]] * scale[page, :, slot // run].astype(np.float64)[:, None]
    return out


def quantised(wl, form: str, run: int):
    """A CPU workload's cache in 8 bits.  Returns (QuantCache of CPU tensors, the
    workload with the dequantised cache).  Scales are powers of two, so that the
    dequantised values are bf16 numbers: the oracle then reads exactly what the
    codes stand for.  Codes of unused slots are NaN (e4m3) or -128 (int8), scales
    of unused runs NaN."""
    codes, scales, plain = [], [], copy.copy(wl)
    for name in ("k_cache", "v_cache"):
        x = getattr(wl, name).float().numpy()
        P, H, Ps, D = x.shape
        runs = x.reshape(P, H, Ps // run, run * D)
        used = ~np.isnan(runs)
        top = np.where(used, np.abs(np.nan_to_num(runs)), 0).max(-1)
        s = np.exp2(np.ceil(np.log2(np.maximum(top, 2.0 ** -100) / TOP[form])))
        code = encode(runs / s[..., None], form)
        value = table(form)[code] * s[..., None]
        code = np.where(used, code, 0x7F if form == "e4m3" else 0x80).astype(np.uint8)
        s = np.where(used.any(-1), s, np.nan).astype(np.float32)
        value = np.where(used, value, np.nan).reshape(x.shape).astype(np.float32)
        codes.append(torch.from_numpy(code.reshape(x.shape)).view(DTYPE[form]))
        scales.append(torch.from_numpy(s))
        bf = torch.from_numpy(value).bfloat16()
        assert torch.equal(torch.nan_to_num(bf.float()), torch.nan_to_num(torch.from_numpy(value)))
        setattr(plain, name, bf)
    return api.QuantCache(*codes, *scales), plain


def to_device(cache, device):
    move = lambda t: t.view(torch.uint8).to(device).view(t.dtype)  # noqa: E731
    return api.QuantCache(move(cache.k), move(cache.v), cache.k_scale.to(device),
                          cache.v_scale.to(device))


def full_attention(q, k, v, scale):
    """q [g][D], k and v [n][D], fp64: (out [g][D], lse [g], a bound on the
    error of each row's scores, which 128 fp32 products and sums, the scales and
    the change of base give)."""
    s = (q @ k.T) * scale
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    mass = p.sum(-1)
    terms = (np.abs(q) @ np.abs(k).T).max(-1) * abs(scale)
    return (p @ v) / mass[:, None], top[:, 0] + np.log(mass), (128 + 8) * 2.0 ** -24 * terms
