"""Plain implementations, on the host, of what the 8-bit KV cache's calls do:
the record's layout and its quantisation, the page bookkeeping row by row,
and attention in 64 bits with a bound on what a kernel may be off.

Bound of an attention output (n tokens, p the exact probabilities, u = 2^-24).
Codes are exact in f16.  Queries are too but for what lies 2^-38 below the
head's largest (scaled so that it is at least 2^14, and f16's last place is
2^-24).  So a logit's products are exact up to that, and its error is that of
an fp32 sum of 128 terms and of three roundings (the scale of the call, the
tile's, their product): dz <= (128 * S + 4 * |z|) * u + 2^-38 * max|q| * K, with
S the sum of the terms' magnitudes and K that of the key's (all scaled), and,
for the rounded difference to the maximum, u * (|z| + |max|) more.  exp2 of
the hardware is good to 2^-22.  Numerator and denominator each change by a
factor within exp(+-dz) * (1 + 2^-22) and are fp32 sums of n terms and,
between steps, waves and splits, some rescalings by exp2 (n + 64 roundings at
most).  p times the tile's scale enters as two f16 parts, each rounded to
nearest: 2^-23 of it.  With A = sum p |v|:
    |out - exact| <= A * (2 * dz + 2 * (n + 64) * u + 2^-20) + T.
T is what the formats cannot hold.  The f16 parts of a product end at 2^-25,
where the scale of the largest V tile so far counts as 2^10 at least: a
token loses at most 2^-35 of that scale times its code, 2^-35 of the largest
|v|.  In fp32 (the open tokens' parts are bf16), a probability relative to
the largest (the denominator is at least 1 there) below 2^-126 may count as
0, and so may a part of its product with the tile's scale, which then
multiplies a code of at most 448: a token loses at most 4 * 2^-126 *
(|v| + 448).  T is the sum of both over the tokens.
"""
import math

import numpy as np

D = 128
Q = {0: 448.0, 1: 127.0}  # SS_KV8_E4M3, SS_KV8_INT8
U = 2.0 ** -24


def record_bytes(blk):
    return 2 * blk * D + 128


def places(blk):
    """Byte of K code (t, c) and of V code (t, c) in a record."""
    k, v = np.zeros((blk, D), np.int64), np.zeros((blk, D), np.int64)
    T = min(blk, 16)
    for token in range(blk):
        s, t = divmod(token, T)
        for c in range(D):
            k[token, c] = s * T * D + (c // 16) * T * 16 + t * 16 + c % 16
            v[token, c] = blk * D + s * T * D + (c % 8 // 4) * T * 64 + (t // 4) * 256 + (c // 8) * 16 + (c % 4) * 4 + t % 4
    return k, v


def code_values(fmt):
    if fmt == 1:
        return np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)
    out = np.zeros(256)
    for x in range(256):
        e, m = (x >> 3) & 15, x & 7
        y = math.nan if (e, m) == (15, 7) else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[x] = -y if x & 128 else y
    return out


def nearest_codes(y, fmt):
    """Codes of fp32 values within the codes' range, rounded to nearest even."""
    if fmt == 1:
        return np.rint(y).astype(np.int32).astype(np.uint8)
    mag = code_values(0)[:127]  # ascending: 0 .. 448
    a = np.abs(y.astype(np.float64))
    hi = np.clip(np.searchsorted(mag, a), 1, 126)
    lo = hi - 1
    dl, dh = a - mag[lo], mag[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (pick | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantise(x, fmt):
    """x float32 [..., blk, d] (bf16 values) -> codes uint8, scale float32 [...], by the header's fp32 steps."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        m = np.maximum(np.abs(x).max((-2, -1)), np.float32(2.0 ** -100))
        ok = np.isfinite(x).all((-2, -1))
        q = np.float32(Q[fmt])
        safe = np.where(ok, m, np.float32(1))
        y = np.where(ok[..., None, None], x, np.float32(0)) * (q / safe)[..., None, None]
        scale = np.where(ok, safe / q, np.float32(np.nan)).astype(np.float32)
    return nearest_codes(y, fmt), scale


def pack(k, v, blk, fmt):
    """Records uint8 [..., rec] of float32 K and V tiles [..., blk, d]."""
    pk, pv = places(blk)
    lead = k.shape[:-2]
    out = np.zeros(lead + (record_bytes(blk),), np.uint8)
    scales = np.zeros(lead + (32,), np.float32)
    for i, (x, at) in enumerate(((k, pk), (v, pv))):
        codes, scales[..., i] = quantise(x, fmt)
        out[..., at.reshape(-1)] = codes.reshape(lead + (-1,))
    out[..., 2 * blk * D:] = np.ascontiguousarray(scales).view(np.uint8)
    return out


def unpack(rec, blk, fmt):
    """float64 K and V tiles [..., blk, d] of records [..., rec]."""
    pk, pv = places(blk)
    values = code_values(fmt)
    scales = np.ascontiguousarray(rec[..., 2 * blk * D:2 * blk * D + 8]).view(np.float32).astype(np.float64)
    lead = rec.shape[:-1]
    tiles = [values[rec[..., at.reshape(-1)]].reshape(lead + (blk, D)) for at in (pk, pv)]
    return tiles[0] * scales[..., 0, None, None], tiles[1] * scales[..., 1, None, None]


def bf16(x):
    """float values rounded to the nearest bf16 (ties to even), as float32; finite."""
    u = np.ascontiguousarray(np.asarray(x, np.float32)).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


# ------------------------------------------------------------- bookkeeping
class Pool:
    """The pages of a batch, row by row."""

    def __init__(self, B, blk, max_blocks, n_pages, free, tables=None, length=None):
        self.B, self.blk, self.max_blocks, self.n_pages = B, blk, max_blocks, n_pages
        self.free = [int(x) for x in free]
        self.tables = np.full((B, max_blocks), -1, np.int32) if tables is None else tables.copy()
        self.len = np.zeros(B, np.int64) if length is None else np.asarray(length, np.int64).copy()

    def held(self, n):
        return -(-n // self.blk)

    def page(self, p):
        return p if 0 <= p < self.n_pages else -1

    def reserve(self, n_new, cap):
        blk = self.blk
        begin, slots, pos = [0], np.full(cap, -1, np.int64), np.full(cap, -1, np.int64)
        taken, status, need_sum, row = [], [], 0, 0
        stack = list(self.free)
        given = 0
        for b in range(self.B):
            n, have = max(0, int(n_new[b])), int(self.len[b])
            taken.append(given)
            end = row + n
            st, need = 0, 0
            if n_new[b] < 0 or have < 0 or (n and end > cap):
                st = 3
            elif self.held(have + n) > self.max_blocks or have + n > 2 ** 31 - 1:
                st = 2
            else:
                need = self.held(have + n) - self.held(have)
                need_sum += need
                if need and need_sum > len(stack):
                    st = 1
            if st == 0:
                for j in range(need):
                    self.tables[b, self.held(have) + j] = self.page(stack[len(stack) - 1 - given - j])
                given += need
                for i in range(n):
                    t = have + i
                    p = self.page(int(self.tables[b, t // blk]))
                    slots[row + i] = p * blk + t % blk if p >= 0 else -1
                    pos[row + i] = t
                self.len[b] = have + n
            status.append(st)
            row = end
            begin.append(min(row, cap))
        self.free = stack[:len(stack) - given]
        return dict(tok_begin=begin, slots=slots, positions=pos, taken=taken + [given], status=status)

    def release(self, done):
        for b in range(self.B):
            if done[b]:
                n = max(0, int(self.len[b]))
                self.free += [self.page(int(p)) for p in self.tables[b, :min(self.held(n), self.max_blocks)]]
                self.len[b] = 0
        del self.free[self.n_pages:]


# --------------------------------------------------------------- attention
def attention(q, k, v, scale):
    """Heads q [G][d] over tokens k, v [n][d] (float64) -> (out, bound) [G][d]."""
    if len(k) == 0:
        return np.zeros(q.shape), np.zeros(q.shape)
    z = q @ k.T * scale
    mag = np.abs(q) @ np.abs(k).T * abs(scale)
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    p /= p.sum(1, keepdims=True)
    dz = ((128 * mag + 4 * np.abs(z) + np.abs(z) + np.abs(m)).max(1, keepdims=True)) * U
    dz += 2.0 ** -38 * np.abs(q).max(1, keepdims=True) * np.abs(k).sum(1).max() * abs(scale)
    lost = len(k) * 2.0 ** -35 * np.abs(v).max() + 4 * 2.0 ** -126 * (np.abs(v) + 448).sum(0)
    return p @ v, (p @ np.abs(v)) * (2 * dz + 2 * (len(k) + 64) * U + 2.0 ** -20) + lost
