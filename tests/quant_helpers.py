"""The 8-bit cache in plain 64-bit arithmetic, for the tests: e4m3 codes with a power-of-two scale per layer, head and
block, pools filled through a block table, storing, and attention with the bounds of its rounding errors."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2512_07993_amd import binding as B

D = 128
U32 = 2.0 ** -24                     # half a step of fp32
U_OUT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def code_values() -> np.ndarray:
    """Value of every e4m3 code (OCP): sign, 4 exponent bits with bias 7, 3 fraction bits; 0x7F and 0xFF are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        x = math.nan if (e, f) == (15, 7) else f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        v[c] = -x if c & 128 else x
    return v


VALUES = code_values()
_POS = VALUES[:127]                  # ascending, 0 .. 448


def encode(x: np.ndarray, byte: int) -> np.ndarray:
    """Codes nearest to x / 2^(byte - 127), ties to the even code, non-finite -> 0x7F.  Needs |x| <= 448 * 2^(byte - 127)."""
    y = np.asarray(x, dtype=np.float64) * 2.0 ** (127 - byte)
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    assert a.max(initial=0.0) <= 448
    hi = np.searchsorted(_POS, a, side="left").clip(max=126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(a == _POS[hi], hi, code)
    code = np.where(np.signbit(y), code | 128, code)
    return np.where(np.isfinite(y), code, 0x7F).astype(np.uint8)


def scale_byte(x: np.ndarray) -> int:
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)].max(initial=0.0)
    if a == 0:
        return 1
    e = math.floor(math.log2(a / 448)) - 2
    while a > 448 * 2.0 ** e:
        e += 1
    return min(max(e + 127, 1), 254)


class Pool:
    """A pool of one kind (K or V) on the host: codes [L, blocks, slots, H, D], bytes [L, H, blocks]."""

    def __init__(self, layers, blocks, slots, heads, fill=0):
        self.codes = np.full((layers, blocks, slots, heads, D), fill, dtype=np.uint8)
        self.byte = np.full((layers, heads, blocks), 127, dtype=np.uint8)

    def store(self, l, h, table, bs, begin, rows):
        """Rows [n, D] at positions begin .. begin + n - 1 of a sequence with block list `table`."""
        t, n = begin, len(rows)
        while t < begin + n:
            p, s = int(table[t // bs]), t % bs
            k = min(bs - s, begin + n - t)
            x = rows[t - begin:t - begin + k]
            byte, old = scale_byte(x), int(self.byte[l, h, p])
            if s > 0:
                byte = max(byte, old)
                if byte > old:
                    was = VALUES[self.codes[l, p, :s, h]] * 2.0 ** (old - 127)
                    self.codes[l, p, :s, h] = encode(was, byte)
            self.byte[l, h, p] = byte
            self.codes[l, p, s:s + k, h] = encode(x, byte)
            t += k

    def rows(self, l, h, table, bs, n):
        t = np.arange(n)
        p = np.asarray(table)[t // bs].astype(np.int64)
        return VALUES[self.codes[l, p, t % bs, h]] * np.exp2(self.byte[l, h, p].astype(np.float64) - 127)[:, None]


def random_table(rng, counts, spare=2, width=None):
    total = int(np.sum(counts)) + spare
    perm = rng.permutation(total)
    table = np.full((len(counts), width or max(1, int(np.max(counts)))), -1, dtype=np.int32)
    at = 0
    for b, k in enumerate(counts):
        table[b, :k] = perm[at:at + k]
        at += k
    return table, total, perm[at:]


def on_device(k: Pool, v: Pool, table, heads_before_slots=False, pad_blocks=0, device="cuda", dtype=torch.uint8):
    """B.QuantCache of two host pools: the plain layout, or [L, blocks, heads, slots, D] seen as the plain one, or with
    unused blocks between the layers."""
    def put(x):
        t = torch.from_numpy(x).to(device)
        if heads_before_slots:
            t = t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
        if pad_blocks:
            big = torch.zeros((t.shape[0], t.shape[1] + pad_blocks) + tuple(t.shape[2:]), dtype=torch.uint8, device=device)
            big[:, :t.shape[1]] = t
            t = big[:, :t.shape[1]]
        return t.view(dtype) if dtype != torch.uint8 else t
    return B.QuantCache(put(k.codes), put(v.codes), torch.from_numpy(k.byte).to(device), torch.from_numpy(v.byte).to(device),
                        torch.from_numpy(np.ascontiguousarray(table)).to(device))


def attend_reference(q, k, v, m, scale, parts, device="cuda"):
    """One (sequence, KV head): q [m, g, D], k and v [n, D] float64 arrays.  Returns out [m, g, D], lse [m, g], and how far
    a result with fp32 sums may be off.

    Bounds, with u = 2^-24: a logit is a sum of 128 exact products (more for an fp32 query's parts) in fp32 and two further
    roundings, so it is off by at most e = (128 + 8) u * scale * sum_d |q_d k_d|; a weight is then off by a factor 1 +- (e + 4u) (the
    power of two is good to one step), and by `parts`: what the weights are rounded to for the second product.  The sums
    over keys add at most one rounding per 32 keys, one per key within a matrix product and lane sum (32), and one per rescaling and
    merge (at most 64): c = (n / 32 + 96) u.  Numerator and denominator together: A * (2 (e + 4u + c) + parts), with
    A = sum_t p_t |v_t|.  The rounding of the output comes on top."""
    t64 = lambda x: torch.as_tensor(np.ascontiguousarray(x), dtype=torch.float64, device=device)
    q, k, v = t64(q), t64(k), t64(v)
    n = k.shape[0]
    g = q.shape[1]
    out = torch.zeros((m, g, D), dtype=torch.float64, device=device)
    lse = torch.full((m, g), -math.inf, dtype=torch.float64, device=device)
    tol = torch.zeros_like(out)
    ltol = torch.zeros_like(lse)
    for j in range(m):
        see = n - m + j + 1
        if see <= 0:
            continue
        kk, vv = k[:see], v[:see]
        s = q[j] @ kk.t() * scale
        e = (128 + 8) * U32 * abs(scale) * (q[j].abs() @ torch.nan_to_num(kk).abs().t()).amax(1)
        c = (see / 32 + 96) * U32
        z = torch.logsumexp(s, 1)
        p = torch.exp(s - z[:, None])
        lse[j], out[j] = z, p @ vv
        a = p @ vv.abs()
        tol[j] = a * (2 * (e[:, None] + 4 * U32 + c) + parts)
        ltol[j] = e + c + 4 * U32 * (2 + z.abs())
    return out.cpu().numpy(), lse.cpu().numpy(), tol.cpu().numpy(), ltol.cpu().numpy()


def check_close(got, ref, tol, what):
    got, ref = np.asarray(got, dtype=np.float64), np.asarray(ref)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref), err_msg="NaN: " + what)
    np.testing.assert_array_equal(np.isinf(got), np.isinf(ref), err_msg="infinities: " + what)
    fin = np.isfinite(ref)
    over = np.abs(got - ref)[fin] - np.broadcast_to(tol, ref.shape)[fin]
    assert over.size == 0 or over.max() <= 0, "%s: beyond its bound by %g (bound %g)" % (what, over.max(), np.broadcast_to(tol, ref.shape)[fin].flat[over.argmax()])
