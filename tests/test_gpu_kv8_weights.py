"""Attention over 8-bit records whose tiles have scales of very different
size: what a tile costs the others goes by its weight in the result, not by
its scale.

Bound.  A logit z_t is off by dz_t, as kv8_ref derives it, token by token; so
the output moves by at most sum p_t dz_t (|v_t| + |out|) and terms of the next
order (2% where the weighted dz is below 2^-7).  exp2, the sums and the two f16
parts have kv8_ref's share.  What the formats cannot hold: a product of a
probability and a V scale, relative to a reference of the kernel's, enters as
two f16 parts whose last place is 2^-24, so it is off by at most 2^-25 (or 2^-23
of itself, which the relative part has).  The largest product so far of the
wave's head is at least 2^10 there.  So a token loses at most 2^-35 of the largest product times its code, which is at most Q:
with p_t the exact probabilities and m_t = Q * scale the largest magnitude of
the token's tile, 2^-35 * max_t(p_t * m_t).  Rescaling is by powers of two.
What fp32 ends at (2^-126 of the largest probability) is as in kv8_ref.
"""
import kv8_ref as ref
import numpy as np
import pytest
from test_gpu_kv8 import D, SCALE, Stored, attend, host, ss  # noqa: F401 -- ss is the fixture

pytestmark = pytest.mark.gpu


def weighed(q, k, v, tile_max):
    """Heads q [G][d] over tokens k, v [n][d] of tiles with these largest magnitudes -> (out, bound) [G][d]."""
    out, _ = ref.attention(q, k, v, SCALE)
    z, mag = q @ k.T * SCALE, np.abs(q) @ np.abs(k).T * SCALE
    m = z.max(1, keepdims=True)
    p = np.exp(z - m)
    p /= p.sum(1, keepdims=True)
    dz = (128 * mag + 5 * np.abs(z) + np.abs(m)) * ref.U
    dz += 2.0 ** -38 * np.abs(q).max(1, keepdims=True) * np.abs(k).sum(1) * SCALE
    lost = len(k) * 2.0 ** -35 * (p * tile_max).max(1, keepdims=True) + 4 * 2.0 ** -126 * (np.abs(v) + 448).sum(0)
    moved = (p * dz) @ np.abs(v) + np.abs(out) * (p * dz).sum(1, keepdims=True)
    return out, 1.02 * moved + (p @ np.abs(v)) * (2 * (len(k) + 64) * ref.U + 2.0 ** -20) + lost


def scale_of(s, g, page, tensor):
    """The fp32 scale of a page's K (0) or V (1) tile, to be written to."""
    at = 2 * s.blk * D + 4 * tensor
    return s.rec[g, page, at:at + 4].view(np.float32)


def check(ss, s, blocks):  # noqa: F811
    """All blocks of every sequence, with one workgroup a unit and with as many as pay."""
    s.k, s.v = ref.unpack(s.rec, s.blk, s.fmt)
    s.to_device()
    for room in (0, None):
        out = host(attend(ss, s, None, blocks, room=room)).astype(np.float64)
        for b in range(s.B):
            for g in range(s.hkv):
                pages = s.tables[b, :s.nblk[b]]
                k, v = s.k[g, pages].reshape(-1, D), s.v[g, pages].reshape(-1, D)
                top = np.repeat(np.array([float(scale_of(s, g, p, 1)[0]) * ref.Q[s.fmt] for p in pages]), s.blk)
                heads = slice(g * s.G, (g + 1) * s.G)
                want, bound = weighed(s.q[b, heads].astype(np.float64), k, v, top)
                off = np.abs(out[b, heads] - want)
                assert (off <= bound).all(), (room, b, g, float((off / bound).max()))


@pytest.mark.parametrize("blk, fmt", [(8, 1), (16, 0), (32, 1)])
@pytest.mark.parametrize("grow", [12, 24, 34, 60, 100])
@pytest.mark.parametrize("where", [0, 37, 63])
def test_a_large_tile_of_no_weight(ss, blk, fmt, grow, where):  # noqa: F811
    """A tile whose V scale is 2^grow times the others' and whose logits lie
    more than 100 below theirs: the others keep their bits."""
    rng = np.random.default_rng(100 * blk + grow + where)
    s = Stored(rng, blk, fmt, [64 * blk, 64 * blk], 2, 4)
    s.q = np.abs(s.q)
    page = s.tables[0, where]
    codes = s.rec[1, page, :blk * D]
    codes[:] = -np.abs(codes.view(np.int8)).view(np.uint8) if fmt else codes | 0x80  # negative keys
    scale_of(s, 1, page, 0)[:] *= np.float32(16)
    scale_of(s, 1, page, 1)[:] *= np.float32(2.0 ** grow)
    check(ss, s, 64)


@pytest.mark.parametrize("blk, fmt", [(8, 0), (16, 1), (32, 0)])
@pytest.mark.parametrize("turn", [-2, -1, 1, 2])
@pytest.mark.parametrize("order", [1, -1])
def test_weights_against_scales(ss, blk, fmt, turn, order):  # noqa: F811
    """Logits that rise (or fall) by about 60 from tile to tile while the V
    scales fall or rise as fast, half or twice as fast: each product counts by
    its own size, whatever came first."""
    rng = np.random.default_rng(7 * blk + turn)
    n = 96
    s = Stored(rng, blk, fmt, [n * blk], 2, 4)
    s.q = np.abs(s.q)
    for g in range(2):
        for j, page in enumerate(s.tables[0, :n][::order]):
            codes = s.rec[g, page, :blk * D]
            codes[:] = np.abs(codes.view(np.int8)).view(np.uint8) if fmt else codes & 0x7F
            values = ref.code_values(fmt)[codes].mean()
            # sum of q * k over the channels, about 60 * j / n in the end
            scale_of(s, g, page, 0)[:] = 60 * j / n / (SCALE * s.q.mean() * values * D)
            scale_of(s, g, page, 1)[:] *= np.float32(2.0 ** (-turn / 2 * 86 * j / n))
    check(ss, s, n)


@pytest.mark.parametrize("blk", [8, 32])
def test_values_near_the_largest(ss, blk):  # noqa: F811
    """Values of one sign up to 2^118, thousands of equal weights: a mean of them, not an infinity."""
    rng = np.random.default_rng(blk)
    s = Stored(rng, blk, 1, [4096], 1, 2)
    s.q *= 0
    codes = s.rec[0, :, blk * D:2 * blk * D].view(np.int8)
    codes[:] = np.abs(codes)
    for page in range(s.n):
        scale_of(s, 0, page, 1)[:] = np.float32(2.0 ** 111)
    check(ss, s, 4096 // blk)


@pytest.mark.parametrize("fmt, G", [(0, 7), (1, 16)])
def test_large_tiles_where_steps_are_shared_out(ss, fmt, G):  # noqa: F811
    """Tables long enough that 512 workgroups share the steps of all sequences,
    each of which has a tile of 2^40 times the others' V scale and no weight."""
    rng = np.random.default_rng(G)
    blk = 32
    s = Stored(rng, blk, fmt, [blk * int(n) for n in rng.integers(1, 60, 14)], 2, G)
    s.q = np.abs(s.q)
    for b in range(1, s.B):
        page = s.tables[b, rng.integers(s.nblk[b])]
        if s.nblk[b] > 1:
            codes = s.rec[b % 2, page, :blk * D]
            codes[:] = -np.abs(codes.view(np.int8)).view(np.uint8) if fmt else codes | 0x80  # negative keys
            scale_of(s, b % 2, page, 0)[:] *= np.float32(16)
            scale_of(s, b % 2, page, 1)[:] *= np.float32(2.0 ** 40)
    check(ss, s, 900)
