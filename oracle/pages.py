"""Oracle: the paged cache of text tokens and its causal attention.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).

The layout of a page is evaluated value by value from its description in include/sali.h; rows are
quantised with the steps of oracle/quant.py, in either 16-bit type; attention is computed in float64
over the rows as they read back.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

GROUP = 32
BLOCK = 16


@dataclass(frozen=True)
class PagesSpec:
    n_kv_heads: int
    n_heads: int
    head_dim: int
    page_tokens: int
    dtype: str            # "fp16" or "bf16"
    store: str            # "16", "int8" or "int4"

    @property
    def half_step(self):
        """Largest relative error of rounding to the 16-bit type."""
        return 2.0 ** -11 if self.dtype == "fp16" else 2.0 ** -8

    @property
    def block_bytes(self):
        d = self.head_dim
        return {"16": 64 * d, "int8": 36 * d, "int4": 22 * d}[self.store]

    @property
    def page_bytes(self):
        return self.block_bytes * (self.page_tokens // BLOCK) * self.n_kv_heads


# ---- 16-bit types as bits --------------------------------------------------------------------------
def to_f32(bits, dtype):
    bits = np.ascontiguousarray(bits, dtype=np.uint16)
    if dtype == "fp16":
        return bits.view(np.float16).astype(np.float32)
    return (bits.astype(np.uint32) << 16).view(np.float32)


def to_bits(x, dtype):
    """fp32 -> 16 bits, nearest even."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    if dtype == "fp16":
        with np.errstate(over="ignore"):
            return x.astype(np.float16).view(np.uint16)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


# ---- the quantiser ---------------------------------------------------------------------------------
def quantise(x, store):
    """fp32 rows [..., D] -> (codes [..., D/32, 32], scale, smallest or None), every step one fp32 operation.  Groups with a value that is not
    finite, or too wide or too small for steps in fp32, become zeros (codes, scale and, where a value is not finite or the group too wide, smallest)."""
    g = x.astype(np.float32).reshape(x.shape[:-1] + (-1, GROUP))
    steps = np.float32(127 if store == "int8" else 15)
    with np.errstate(all="ignore"):
        if store == "int8":
            low, m = None, np.abs(g).max(-1)
        else:
            low = g.min(-1)
            m = (g.max(-1) - low).astype(np.float32)
            g = (g - low[..., None]).astype(np.float32)
        sound = np.isfinite(x.reshape(g.shape)).all(-1) & np.isfinite(m)
        inv = (steps / m).astype(np.float32)
        some = sound & (m > 0) & np.isfinite(inv)
        scale = np.where(some, m / steps, 0).astype(np.float32)
        q = np.where(some[..., None], np.clip(np.rint((g * inv[..., None]).astype(np.float32)), -127 if store == "int8" else 0, steps), 0)
        if low is not None:
            low = np.where(sound, low, 0).astype(np.float32)
    return q.astype(np.int32), scale, low


def read_back(bits, spec):
    """The rows (16-bit patterns [..., D]) that rows of these bits read back as."""
    if spec.store == "16":
        return np.array(bits, dtype=np.uint16)
    q, scale, low = quantise(to_f32(bits, spec.dtype), spec.store)
    x = q.astype(np.float64) * scale[..., None]
    if low is not None:
        x = x + low[..., None]
    return to_bits(x.astype(np.float32), spec.dtype).reshape(np.shape(bits))


# ---- layout ----------------------------------------------------------------------------------------
def place(t):
    a, b, i = t // 8, t // 4 % 2, t % 4
    return 8 * b + 4 * a + i


def _parts(spec):
    d = spec.head_dim
    code = {"16": 32 * d, "int8": 16 * d, "int4": 8 * d}[spec.store]
    scale = 0 if spec.store == "16" else 2 * d
    zero = d if spec.store == "int4" else 0
    return np.cumsum([0, code, code, scale, scale, zero, zero])


def byte_of(spec, side, t, e):
    """(offset in its block, shift in bits) of value e of token t; side 0 = K, 1 = V."""
    d, at, p = spec.head_dim, _parts(spec)[side], place(t)
    if spec.store == "16":
        return at + (((e // 8 * 16 + p) * 8 + e % 8) * 2 if side == 0 else ((t // 8 * d + e) * 8 + t % 8) * 2), 0
    if spec.store == "int8":
        return at + ((e // 16 * 16 + p) * 16 + e % 16 if side == 0 else (t // 8 * d + e) * 8 + t % 8), 0
    g, w = e // 32, e % 32
    return at + ((g * 16 + p) * 16 + w % 16 if side == 0 else ((t // 8 * (d // 32) + g) * 16 + w % 16) * 8 + t % 8), 4 * (w // 16)


def block_bytes_of(spec, k_bits, v_bits, block, own):
    """`block` (uint8, a copy is returned) with the rows k_bits, v_bits [16, D] of the tokens `own` put in."""
    block = np.array(block, dtype=np.uint8)
    parts, d = _parts(spec), spec.head_dim
    for side, bits in ((0, k_bits), (1, v_bits)):
        if spec.store == "16":
            codes = bits
        else:
            codes, scale, low = quantise(to_f32(bits, spec.dtype), spec.store)
            codes = codes.reshape(BLOCK, d)
        for t in own:
            for e in range(d):
                at, shift = byte_of(spec, side, t, e)
                if spec.store == "16":
                    block[at], block[at + 1] = int(codes[t, e]) & 255, int(codes[t, e]) >> 8
                elif spec.store == "int8":
                    block[at] = int(codes[t, e]) & 255
                else:
                    block[at] = (int(block[at]) & (0xF0 if shift == 0 else 0x0F)) | int(codes[t, e]) << shift
            for g in range(0 if spec.store == "16" else d // GROUP):
                at = parts[2 + side] + (g * 16 + (place(t) if side == 0 else t)) * 4
                block[at:at + 4] = np.frombuffer(np.float32(scale[t, g]).tobytes(), np.uint8)
                if spec.store == "int4":
                    at = parts[4 + side] + (g * 16 + (place(t) if side == 0 else t)) * 2
                    block[at:at + 2] = np.frombuffer(to_bits(low[t, g:g + 1], spec.dtype).tobytes(), np.uint8)
    return block


# ---- attention -------------------------------------------------------------------------------------
def attend(q, k, v, length, scale, window=0, sinks=0, prior=None, prior_lse=None, hidden=None):
    """One sequence: q [n, n_heads, D], k, v [length, n_kv, D] (float64) -> out [n, n_heads, D], lse [n, n_heads], and, for error bounds,
    weights' sum over |V| and the largest sum of |q k|, alike.  hidden: positions that nobody sees (pages that are none)."""
    n, hq, d = q.shape
    group = hq // k.shape[1]
    pos = np.arange(length - n, length)[:, None]
    j = np.arange(length)[None]
    seen = j <= pos
    if window > 0:
        seen &= (j > pos - window) | (j < sinks)
    if hidden is not None:
        seen &= ~hidden[None, :length]
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -np.inf)
    mass, reach = np.zeros((n, hq, d)), np.zeros((n, hq))
    for h in range(hq):
        kh, vh = k[:length, h // group], v[:length, h // group]
        with np.errstate(all="ignore"):
            s = np.where(seen, scale * (q[:, h] @ kh.T), -np.inf)
            top = np.where(seen.any(1), s.max(1, initial=-np.inf), 0.0)[:, None]
            p = np.where(seen, np.exp(s - top), 0.0)
            total = p.sum(1)
            ok = total != 0
            w = np.where(ok[:, None], p / np.where(ok, total, 1.0)[:, None], 0.0)
            lse[:, h] = np.where(ok, top[:, 0] + np.log(np.where(ok, total, 1.0)), -np.inf)
            # a key out of sight does not reach the row, whatever its value
            for t in range(n):
                out[t, h] = w[t, seen[t]] @ vh[seen[t]]
                mass[t, h] = w[t, seen[t]] @ np.abs(vh[seen[t]])
            reach[:, h] = np.where(seen, np.abs(scale) * (np.abs(q[:, h]) @ np.abs(kh).T), 0.0).max(1, initial=0.0)
    if prior is not None:
        with np.errstate(all="ignore"):
            both = np.logaddexp(lse, prior_lse)
            own = np.where(np.isneginf(lse), 0.0, np.exp(lse - both))[..., None]
            other = np.where(np.isneginf(prior_lse), 0.0, np.exp(prior_lse - both))[..., None]
            out = np.where(own > 0, own * out, 0.0) + np.where(other > 0, other * prior, 0.0)
            mass = own * mass + np.where(other > 0, other * np.abs(prior), 0.0)
        lse = both
    return out, lse, mass, reach


def bounds(spec, out, lse, mass, reach, length, v_max):
    """How far a right result may be from `attend`'s, elementwise: (out, lse).  Every step at its worst:
    the D products of a score are summed in fp32, D 2^-24 of the sum of their sizes (reach); scaling and the subtraction of the
    reference, 2^-23 of the score's and reference's sizes, both within reach, once for the row and once for where a reference moves; exp2,
    log2 and divisions, 2^-21 in all; sums over the keys and over partial results in fp32, (keys + 64) 2^-24.  These all move a weight
    relative to the others: `step`.  Weights are rounded to 16 bits for the product with V (half a step; fp16: 2^-35 of the largest at the least,
    since it is 2^10 or more where weights are rounded and fp16's smallest step is 2^-24), the result once more."""
    u = spec.half_step
    step = reach * (spec.head_dim * 2.0 ** -24 + 4 * 2.0 ** -23) + 2.0 ** -21 + (length + 64) * 2.0 ** -24
    d_out = 1.01 * ((2 * step[..., None] + u) * mass + u * np.abs(out)) + 2.0 ** -24
    if spec.dtype == "fp16":
        d_out = d_out + length * 2.0 ** -35 * v_max
    d_lse = step + 2.0 ** -22 * (1.0 + np.where(np.isfinite(lse), np.abs(lse), 0.0))
    return d_out, d_lse
