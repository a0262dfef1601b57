"""The 8-bit KV cache on the GPU against the plain implementations of
kv8_ref: page bookkeeping and stored codes exactly, attention within the
bound derived there; then the calls together, as a serving step makes them."""
import math

import kv8_ref as ref
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1.0 / math.sqrt(D)


@pytest.fixture(scope="module")
def ss():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2509_24626_amd import binding
    binding.lib()
    return binding


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype))).cuda()


def empty(*shape, fill=-77, dtype=torch.int32):
    return torch.full(shape, fill, dtype=dtype, device="cuda")


def host(t):
    return t.cpu().numpy()


def to_bf16(a):
    """bf16 tensor of float32 values that bf16 holds."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).cuda()


# ------------------------------------------------------------ block tables
class Tables:
    """The device side of a pool, each call beside the model's."""

    def __init__(self, ss, B, blk, max_blocks, n_pages, rng, n_free=None, in_place=True):
        self.ss, self.B, self.blk, self.max_blocks, self.n_pages, self.in_place = ss, B, blk, max_blocks, n_pages, in_place
        free = rng.permutation(n_pages)[:n_pages if n_free is None else n_free]
        self.model = ref.Pool(B, blk, max_blocks, n_pages, free)
        stack = np.full(n_pages, -5)
        stack[:len(free)] = free
        self.free, self.n_free = dev(stack), dev([len(free)])
        self.tables, self.len = dev(self.model.tables), dev(self.model.len)
        self.nblk = empty(B)

    def _outs(self):
        return (self.len, self.n_free) if self.in_place else (empty(self.B), empty(1))

    def reserve(self, n_new, cap, positions=True, offset=0, check=True):
        rows = lambda: empty(cap + 8)[offset:offset + cap]  # noqa: E731 -- any 4-byte alignment
        slots, pos = rows(), rows() if positions else None
        begin, taken, status = empty(self.B + 1), empty(self.B + 1), empty(self.B)
        len_out, n_free_out = self._outs()
        self.ss.ss_block_tables(self.len, dev(n_new), self.n_free, self.B, self.blk, self.max_blocks, self.n_pages,
                                self.free, self.tables, len_out, self.nblk, n_free_out, begin, slots, pos, cap, taken,
                                status)
        self.len, self.n_free = len_out, n_free_out
        if check:
            want = self.model.reserve(n_new, cap)
            got = dict(tok_begin=begin, slots=slots, taken=taken, status=status)
            if positions:
                got["positions"] = pos
            for name, t in got.items():
                assert np.array_equal(host(t), want[name]), name
            self.same()
        return begin, slots, pos, status

    def release(self, done, check=True):
        len_out, n_free_out = self._outs()
        self.ss.ss_block_release(self.len, dev(done), self.n_free, self.B, self.blk, self.max_blocks, self.n_pages,
                                 self.tables, self.free, len_out, self.nblk, n_free_out)
        self.len, self.n_free = len_out, n_free_out
        if check:
            self.model.release(done)
            self.same()

    def same(self):
        m = self.model
        assert np.array_equal(host(self.len), m.len)
        assert np.array_equal(host(self.nblk), np.maximum(m.len, 0) // self.blk)
        assert host(self.n_free)[0] == len(m.free)
        assert np.array_equal(host(self.free)[:len(m.free)], m.free)
        assert np.array_equal(host(self.tables), m.tables)


@pytest.mark.parametrize("B, blk, longest, in_place", [
    (1, 16, 3, True), (1, 8, 9000, False), (2, 32, 5000, True), (63, 16, 40, True), (64, 8, 1, False),
    (65, 32, 700, True), (200, 16, 90, False), (1000, 8, 12, True), (1025, 16, 3, True), (1500, 8, 30, False),
    (4100, 8, 40, True), (9000, 16, 5, False)])
def test_tables_over_several_steps(ss, B, blk, longest, in_place):
    """Rows that join, grow, idle and finish over five steps of every length
    up to `longest`, with one launch (up to 4096 token rows) and with two."""
    rng = np.random.default_rng(B * 100 + blk)
    max_blocks = 6 * (longest // blk + 2)
    t = Tables(ss, B, blk, max_blocks, B * max_blocks // 2 + 7, rng, in_place=in_place)
    for step in range(5):
        n = rng.integers(0, longest + 1, B)
        n[rng.random(B) < 0.3] = 0
        cap = int(n.sum()) + int(rng.integers(0, 70))
        t.reserve(n, cap, positions=step != 1, offset=step % 4)
        t.release((rng.random(B) < 0.35).astype(np.int32))
    t.release(np.ones(B))
    assert host(t.n_free)[0] == t.n_pages


@pytest.mark.parametrize("cap", [200, 5000])
def test_tables_rows_that_are_not_served(ss, cap):
    """A pool that runs out, a row past its table, a negative length, negative
    and huge counts, and token rows past token_cap: each row's status, and
    nothing taken by rows that are not served."""
    rng = np.random.default_rng(11)
    t = Tables(ss, 9, 16, 4, 40, rng, n_free=9)
    t.reserve([5, 16, 0, 30, 64, 0, 0, 0, 0], cap)  # the last needs more than is left
    t.reserve([60, 0, 1, 0, 0, 2 ** 31 - 1, 0, 0, 0], cap)  # past the table; past token_cap with all behind
    t.reserve([1, 65, -3, 1, 17, 17, 1, 0, 1], cap)
    t.model.len[2] = -4
    t.len.copy_(dev(t.model.len))
    t.reserve([1, 1, 1, 1, 1, 1, 1, 1, 1], cap)
    t.reserve([3, 3, 0, 3, 3, cap, 3, 0, 3], cap)


def test_tables_row_sums_past_32_bits(ss):
    rng = np.random.default_rng(12)
    t = Tables(ss, 70, 8, 8, 100, rng)
    t.reserve([3] + [2 ** 31 - 1] * 68 + [2], 64)


@pytest.mark.parametrize("cap", [64, 5000])
def test_tables_of_rows_near_the_largest_length(ss, cap):
    """A length grows up to 2^31 - 1 and never past it."""
    blk, top = 32, 2 ** 31 - 1
    max_blocks = top // blk + 2  # so that the table is not what ends it
    tables = empty(2, max_blocks, fill=3)
    ln, nblk, n_free = dev([top - 8, top - 29]), empty(2), dev([4])
    begin, taken, status, slots, pos = empty(3), empty(3), empty(2), empty(cap), empty(cap)
    ss.ss_block_tables(ln, dev([20, 29]), n_free, 2, blk, max_blocks, 8, dev(np.arange(8)), tables, ln, nblk, n_free, begin,
                       slots, pos, cap, taken, status)
    assert host(status).tolist() == [2, 0] and host(ln).tolist() == [top - 8, top] and host(n_free)[0] == 4
    assert host(begin).tolist() == [0, 20, 49] and host(taken).tolist() == [0, 0, 0]
    assert host(nblk).tolist() == [(top - 8) // blk, top // blk]
    where = np.concatenate([np.full(20, -1), np.arange(top - 29, top), np.full(cap - 49, -1)])
    assert np.array_equal(host(pos), where)
    assert np.array_equal(host(slots), np.where(where < 0, -1, 3 * blk + where % blk))
    assert bool((tables == 3).all())


def test_tables_bad_page_numbers(ss):
    """Page numbers outside the pool give slots of -1 and never an address."""
    rng = np.random.default_rng(13)
    t = Tables(ss, 3, 8, 10, 20, rng)
    t.reserve([5, 8, 3], 32)
    for where, bad in ((0, 20), (2, -9)):
        t.model.tables[where, 0] = bad
    t.tables.copy_(dev(t.model.tables))
    t.model.free[-2:] = [2 ** 30, -1]
    t.free[:len(t.model.free)] = dev(t.model.free)
    t.reserve([9, 9, 1], 32)
    t.release([1, 0, 1])


def test_release_of_large_tables(ss):
    """Rows of several thousand pages, more than one workgroup copies."""
    rng = np.random.default_rng(14)
    t = Tables(ss, 5, 8, 5000, 20000, rng)
    t.reserve([39999, 1, 17000, 0, 33000], 100000)
    t.release([1, 0, 0, 1, 1])
    t.release([0, 1, 1, 0, 0])


# ------------------------------------------------------------------- write
def open_tiles(o, B, hkv, blk):
    """K and V [B][Hkv][blk][d] of open records."""
    o = o.reshape(B, hkv, 2, blk * D)
    return o[:, :, 0].reshape(B, hkv, blk, D), o[:, :, 1].reshape(B, hkv, D, blk).transpose(0, 1, 3, 2)


def open_records(k, v):
    B, hkv, blk, _ = k.shape
    return np.concatenate([k.reshape(B, hkv, -1), v.transpose(0, 1, 3, 2).reshape(B, hkv, -1)], -1)


def values(rng, *shape):
    """bf16 values of mixed magnitudes, as float32."""
    return ref.bf16(rng.standard_normal(shape) * np.exp2(rng.integers(-6, 7, shape[:-1] + (1,))))


class Written:
    """A write call and what it should leave."""

    def __init__(self, ss, rng, blk, fmt, meta, length, n_new, hkv=3, layout="fused", extra=3, unserved=()):
        self.ss, self.blk, self.fmt, self.meta_kind, self.hkv = ss, blk, fmt, meta, hkv
        B = self.B = len(length)
        n = int(np.sum(n_new))
        cap = n + extra
        self.length, self.n_new = np.asarray(length), np.asarray(n_new)
        begin = np.concatenate([[0], np.cumsum(n_new)])
        blocks = -(-(self.length + self.n_new) // blk)
        self.n_pages = int(blocks.sum()) + 4
        pages = rng.permutation(self.n_pages)
        at = np.cumsum(blocks) - blocks
        slots, pos = np.full(cap, -1), np.full(cap, -1)
        for b in range(B):
            for i in range(int(n_new[b])):
                p = self.length[b] + i
                pos[begin[b] + i] = p
                slots[begin[b] + i] = -1 if b in unserved else pages[at[b] + p // blk] * blk + p % blk
        self.k, self.v = values(rng, cap, hkv, D), values(rng, cap, hkv, D)
        self.open_k, self.open_v = values(rng, B, hkv, blk, D), values(rng, B, hkv, blk, D)
        self.nblk_max = max(1, int((blocks - 1).max()))  # one block fewer than some sequence reaches
        self.expect(begin, slots, pos, unserved)
        rec = ref.record_bytes(blk)
        self.records = empty(hkv, self.n_pages, rec, fill=0x5A, dtype=torch.uint8)
        self.region = dev(np.tile(np.arange(hkv) * self.n_pages * rec, B), np.int64)
        self.open = to_bf16(open_records(self.open_k, self.open_v))
        per = {None: 0, 0: 2 * D, 1: D}[meta]
        self.meta = empty(B, hkv, self.nblk_max, per, fill=7.0, dtype=torch.bfloat16) if per else None
        kv = torch.empty(0)
        if layout == "fused":  # [token][head][2][d]
            kv = to_bf16(np.stack([self.k, self.v], 2))
            base, args = kv.data_ptr(), (hkv * 4 * D, 4 * D)
            kp, vp = base, base + 2 * D
        elif layout == "planes":  # [2][head][token][d]
            kv = to_bf16(np.stack([self.k.transpose(1, 0, 2), self.v.transpose(1, 0, 2)]))
            kp, vp, args = kv.data_ptr(), kv[1].data_ptr(), (2 * D, cap * 2 * D)
        else:  # a slice of a wider projection: [token][head][d + 8]
            kv = to_bf16(np.concatenate([np.stack([self.k, self.v]), np.full((2, cap, hkv, 8), 3e38)], -1))
            kp, vp, args = kv.data_ptr(), kv[1].data_ptr(), (hkv * 2 * (D + 8), 2 * (D + 8))
        self.args = (kp, vp, *args, dev(begin), dev(slots), dev(pos), B, hkv, blk, D, cap, fmt, self.records, self.region,
                     self.n_pages, self.open, self.meta, meta or 0, self.nblk_max)
        self.kv = kv

    def expect(self, begin, slots, pos, unserved):
        blk, fmt = self.blk, self.fmt
        self.want_records = {}  # page -> [head][rec]
        self.want_meta = {}  # (b, j) -> K tile [head][blk][d]
        self.want_k, self.want_v = self.open_k.copy(), self.open_v.copy()
        for b in range(self.B):
            if b in unserved:
                continue
            i0, n, p0 = int(begin[b]), int(self.n_new[b]), int(self.length[b]) % blk
            k = np.concatenate([self.open_k[b, :, :p0], self.k[i0:i0 + n].transpose(1, 0, 2)], 1)
            v = np.concatenate([self.open_v[b, :, :p0], self.v[i0:i0 + n].transpose(1, 0, 2)], 1)
            full = k.shape[1] // blk
            for m in range(full):
                kt, vt = k[:, m * blk:(m + 1) * blk], v[:, m * blk:(m + 1) * blk]
                page = int(slots[i0 + (m + 1) * blk - p0 - 1]) // blk
                self.want_records[page] = ref.pack(kt, vt, blk, fmt)
                self.want_meta[b, int(self.length[b]) // blk + m] = kt
            rest, lo = k.shape[1] - full * blk, 0 if full else p0
            self.want_k[b, :, lo:rest] = k[:, full * blk + lo:]
            self.want_v[b, :, lo:rest] = v[:, full * blk + lo:]

    def run(self):
        self.ss.ss_write_kv8(*self.args)

    def check(self):
        got = host(self.records)
        for page in range(self.n_pages):
            want = self.want_records.get(page, np.full(got[:, 0].shape, 0x5A))
            assert np.array_equal(got[:, page], want), page
        k, v = open_tiles(self.open.float().cpu().numpy(), self.B, self.hkv, self.blk)
        assert np.array_equal(k, self.want_k) and np.array_equal(v, self.want_v)
        if self.meta is None:
            return
        meta = self.meta.float().cpu().numpy()
        for b in range(self.B):
            for j in range(self.nblk_max):
                tile = self.want_meta.get((b, j))
                if tile is None:
                    assert (meta[b, :, j] == 7.0).all()
                elif self.meta_kind == 0:
                    assert np.array_equal(meta[b, :, j], np.concatenate([tile.min(1), tile.max(1)], -1))
                else:  # the fp64 mean, rounded once
                    mean = tile.astype(np.float64).mean(1)
                    assert np.array_equal(meta[b, :, j], round_once(mean))


def round_once(x):
    """float64 to bf16, one rounding (nearest even), as float32; normal range."""
    e = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 1e-300))) - 7)
    return (np.rint(x / e) * e).astype(np.float32)


SHAPES = [  # lengths held, new tokens, for blocks of t
    lambda t: ([0], [1]), lambda t: ([t - 1], [1]), lambda t: ([3 * t + 2], [t - 2]), lambda t: ([0], [5 * t + 3]),
    lambda t: ([t // 2], [4 * t]),
    lambda t: ([0, t - 1, 7, 2 * t, 2 * t + 1, 0, 5], [0, 1, 0, 2 * t, t - 1, 3, 3 * t - 5]),
    lambda t: ([b % t for b in range(70)], [1] * 70), lambda t: ([0] * 37 + [4], [0] * 37 + [2 * t])]


@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_write(ss, blk, fmt, shape):
    """Codes, scales, open rows and metadata of every length around a block's
    end; pages, rows and metadata that are not the call's keep their bytes."""
    rng = np.random.default_rng(1000 * blk + 10 * shape + fmt)
    meta, layout = [None, 0, 1][(shape + fmt) % 3], ["fused", "planes", "wide"][shape % 3]
    length, n_new = SHAPES[shape](blk)
    w = Written(ss, rng, blk, fmt, meta, length, n_new, hkv=[3, 1, 8, 2][shape % 4], layout=layout)
    w.run()
    w.check()


@pytest.mark.parametrize("blk", [8, 16, 32])
def test_write_leaves_rows_without_pages_out(ss, blk):
    rng = np.random.default_rng(blk)
    w = Written(ss, rng, blk, 0, 0, [3, 5, 0], [2 * blk, 3 * blk, blk + 1], unserved=(1,))
    w.run()
    w.check()


def test_write_of_pages_out_of_range(ss):
    """A page at or past slot_limit is not written; the others are."""
    rng = np.random.default_rng(21)
    w = Written(ss, rng, 16, 1, None, [0], [64])
    pages = sorted(w.want_records)
    a = list(w.args)
    a[15] = pages[-1]  # slot_limit: the highest page falls out
    w.ss.ss_write_kv8(*a)
    del w.want_records[pages[-1]]
    w.check()


@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("fmt", [0, 1])
def test_write_rounds_to_nearest_even(ss, blk, fmt):
    """Tiles whose largest magnitude is Q, so that codes are the rounded
    values: every bf16 in the codes' range and on either side of their ties."""
    rng = np.random.default_rng(22)
    bits = np.arange(0x3A00, 0x43E1 if fmt == 0 else 0x42FF, dtype=np.uint32)  # 2^-11 .. Q
    v = (bits << 16).astype(np.uint32).view(np.float32)
    v = np.concatenate([v, -v, [0.0, -0.0]]).astype(np.float32)
    v = np.concatenate([rng.permutation(v), np.zeros(-len(v) % (blk * D - 1), np.float32)]).reshape(-1, blk * D - 1)
    tiles = np.concatenate([np.full((len(v), 1), ref.Q[fmt], np.float32), v], 1).reshape(-1, blk, D)
    n = len(tiles)
    w = Written(ss, rng, blk, fmt, None, [0] * n, [blk] * n, hkv=1, extra=0)
    w.k = w.v = tiles.reshape(n * blk, 1, D)
    w.kv.copy_(to_bf16(np.stack([w.k, w.v], 2)))
    w.expect(*(host(t) for t in w.args[4:7]), ())
    w.run()
    w.check()
    assert (host(w.records)[0, :, 2 * blk * D:2 * blk * D + 8].copy().view(np.float32)[sorted(w.want_records)] == 1.0).all()


@pytest.mark.parametrize("fmt", [0, 1])
def test_write_of_extreme_tiles(ss, fmt):
    """Zeros, subnormal and largest magnitudes; a tile with an infinity or a
    NaN gets the scale NaN and codes 0, alone of its block's two."""
    rng = np.random.default_rng(23)
    blk, n = 16, 6
    w = Written(ss, rng, blk, fmt, None, [0] * n, [blk] * n, hkv=1, extra=0)
    w.k[:blk], w.v[:blk] = 0.0, -0.0
    w.k[blk:2 * blk], w.v[blk:2 * blk] = ref.bf16(w.k[blk:2 * blk] * 1e-41), ref.bf16(w.v[blk:2 * blk] * 1e-29)
    w.k[2 * blk:3 * blk] = np.sign(w.k[2 * blk:3 * blk]) * ref.bf16(3.3e38)
    w.k[3 * blk + 5, 0, 77] = np.inf
    w.v[4 * blk + 15, 0, 0] = np.nan
    w.v[5 * blk, 0, 127] = -np.inf
    w.kv.copy_(to_bf16(np.stack([w.k, w.v], 2)))
    w.expect(*(host(t) for t in w.args[4:7]), ())
    w.run()
    got, pages = host(w.records)[0], host(w.args[5])[blk - 1::blk] // blk
    for i, page in enumerate(pages):
        want = w.want_records[page][0]
        assert np.array_equal(got[page, :2 * blk * D], want[:2 * blk * D]), i
        a, b = (r[2 * blk * D:2 * blk * D + 8].copy().view(np.float32) for r in (got[page], want))
        assert np.array_equal(a, b, equal_nan=True)
        assert np.isnan(a).tolist() == [i == 3, i in (4, 5)]


@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("kind", [0, 1])
def test_write_metadata_is_that_of_the_bf16_records(ss, blk, kind):
    """The metadata beside the codes, signed zeros included, equals that of
    ss_build_metadata(_mean) over the same blocks as bf16 records."""
    rng = np.random.default_rng(24)
    n, hkv = 9, 2
    w = Written(ss, rng, blk, 0, kind, [0], [n * blk + 3], hkv=hkv)
    w.k[rng.random(w.k.shape) < 0.3] = -0.0
    w.k[rng.random(w.k.shape) < 0.2] = 0.0
    w.kv.copy_(to_bf16(np.stack([w.k, w.v], 2)))
    w.run()
    kt = w.k[:n * blk].reshape(n, blk, hkv, D).transpose(2, 0, 1, 3)
    recs = to_bf16(open_records(kt, kt))  # [head][block][2*blk*d]
    off = dev(np.arange(hkv) * n * 4 * blk * D, np.int64)
    want = torch.empty_like(w.meta)
    build = ss.ss_build_metadata if kind == 0 else ss.ss_build_metadata_mean
    build(recs, off, dev([n]), 1, hkv, w.nblk_max, blk, D, want)
    assert torch.equal(w.meta[:, :, :n].view(torch.int16), want[:, :, :n].view(torch.int16))


# -------------------------------------------------------------- stored state
class Stored:
    """A pool of records and everything around it."""

    def __init__(self, rng, blk, fmt, length, hkv, G, paged=True, spare=4):
        self.blk, self.fmt, self.hkv, self.G = blk, fmt, hkv, G
        self.len = np.asarray(length)
        B = self.B = len(length)
        self.nblk = self.len // blk
        held = -(-self.len // blk)
        self.max_blocks = max(1, int(held.max()) + 1)
        self.n = int(held.sum()) + spare
        pages = rng.permutation(self.n)
        self.tables = np.full((B, self.max_blocks), -1)
        at = np.cumsum(held) - held
        for b in range(B):
            self.tables[b, :held[b]] = pages[at[b]:at[b] + held[b]]
        s = ref.bf16(0.5 + 1.5 * rng.random((hkv, 1, 1, D)))
        tile = lambda: ref.bf16(rng.standard_normal((hkv, self.n, blk, D)) * s)  # noqa: E731
        self.rec = ref.pack(tile(), tile(), blk, fmt)
        self.k, self.v = ref.unpack(self.rec, blk, fmt)
        self.open_k, self.open_v = values(rng, B, hkv, blk, D), values(rng, B, hkv, blk, D)
        self.q = ref.bf16(rng.standard_normal((B, hkv * G, D)))

    def to_device(self):
        rec = ref.record_bytes(self.blk)
        self.d_rec = torch.from_numpy(self.rec).cuda()
        self.d_region = dev(np.tile(np.arange(self.hkv) * self.n * rec, self.B), np.int64)
        self.d_tables, self.d_len, self.d_nblk = dev(self.tables), dev(self.len), dev(self.nblk)
        self.d_open = to_bf16(open_records(self.open_k, self.open_v))
        self.d_q = to_bf16(self.q)
        return self

    def tokens(self, b, g, entries, open_rows):
        """K and V (float64) of block entries of sequence b, then open rows."""
        pages = [self.tables[b, e] for e in entries if 0 <= e < min(self.max_blocks, self.nblk[b])]
        k = [self.k[g, p] for p in pages if 0 <= p < self.n] + [self.open_k[b, g, :open_rows]]
        v = [self.v[g, p] for p in pages if 0 <= p < self.n] + [self.open_v[b, g, :open_rows]]
        return np.concatenate(k).astype(np.float64), np.concatenate(v).astype(np.float64)

    def check(self, out, entries, with_open):
        """out [B][Hq][d] against the plain attention; entries(b, g) -> block list."""
        out, worst = host(out).astype(np.float64), 0.0
        for b in range(self.B):
            for g in range(self.hkv):
                k, v = self.tokens(b, g, entries(b, g), int(self.len[b]) % self.blk if with_open else 0)
                heads = slice(g * self.G, (g + 1) * self.G)
                want, bound = ref.attention(self.q[b, heads].astype(np.float64), k, v, SCALE)
                assert (np.abs(out[b, heads] - want) <= bound).all(), (b, g, np.abs(out[b, heads] - want).max(), bound.min())
                worst = max(worst, float(np.abs(out[b, heads] - want).max()))
        return worst


def attend(ss, s, sel=None, k=None, with_open=False, tables=True, nblk=True, capacity=None, limit=None, room=None,
           rec=None, region=None, q=None, stream=None):
    k = sel.shape[-1] if sel is not None else k
    need = ss.ss_sparse_attention_kv8_workspace(s.B, s.hkv * s.G, s.hkv, D, s.blk, k) if room is None else room
    ws = empty(max(need, 16), fill=0xFF, dtype=torch.uint8) if need else None  # NaN partials
    out = empty(s.B, s.hkv * s.G, D, fill=float("nan"), dtype=torch.float32)
    ss.ss_sparse_attention_kv8(s.d_q if q is None else q, s.d_rec if rec is None else rec,
                               s.d_region if region is None else region, None if sel is None else dev(sel),
                               s.d_tables if tables else None, s.max_blocks if tables else 0, capacity,
                               s.n if limit is None else limit, s.d_nblk if nblk else None,
                               s.d_open if with_open else None, s.d_len if with_open else None, s.fmt, s.B,
                               s.hkv * s.G, s.hkv, D, s.blk, k, SCALE, out, ws, need, stream)
    return out


# -------------------------------------------------------------------- read
@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("layout", ["fused", "planes"])
def test_read(ss, blk, fmt, layout):
    """Whole histories, prefixes, more rows than a sequence holds, none, and
    rows past the buffer's; values are code * scale in fp32, rounded once."""
    rng = np.random.default_rng(31 + blk)
    hkv = 3
    length = [0, 1, blk - 1, blk, 5 * blk + 3, 4 * blk, 2 * blk + 1]
    want_rows = [0, 1, blk - 1, blk, 5 * blk + 3, 2 * blk + 3, 3 * blk]
    s = Stored(rng, blk, fmt, length, hkv, 1).to_device()
    s.tables[4, 2] = s.n  # out of range: reads as zeros
    s.d_tables = dev(s.tables)
    begin = np.concatenate([[0], np.cumsum(want_rows)])
    rows = int(begin[-1]) - 2
    if layout == "fused":
        out = empty(rows + 4, hkv, 2, D, fill=9.0, dtype=torch.bfloat16)
        k, v, strides = out.data_ptr(), out.data_ptr() + 2 * D, (hkv * 4 * D, 4 * D)
        gk, gv = out[:, :, 0], out[:, :, 1]
    else:
        out = empty(2, hkv, rows + 4, D, fill=9.0, dtype=torch.bfloat16)
        k, v, strides = out.data_ptr(), out[1].data_ptr(), (2 * D, (rows + 4) * 2 * D)
        gk, gv = out[0].transpose(0, 1), out[1].transpose(0, 1)
    ss.ss_read_kv8(s.d_rec, s.d_region, s.d_tables, s.max_blocks, s.n, s.d_open, s.d_len, dev(begin), s.B, hkv, blk, D,
                   rows, fmt, k, v, *strides)
    wk, wv = np.full((rows + 4, hkv, D), 9.0, np.float32), np.full((rows + 4, hkv, D), 9.0, np.float32)
    k32, v32 = s.k.astype(np.float32), s.v.astype(np.float32)  # codes * scale: one fp32 rounding of the exact product
    for b in range(s.B):
        for t in range(min(want_rows[b], length[b])):
            r = begin[b] + t
            if r >= rows:
                continue
            if t // blk < s.nblk[b]:
                p = s.tables[b, t // blk]
                wk[r] = ref.bf16(k32[:, p, t % blk]) if p < s.n else 0
                wv[r] = ref.bf16(v32[:, p, t % blk]) if p < s.n else 0
            else:
                wk[r], wv[r] = s.open_k[b, :, t % blk], s.open_v[b, :, t % blk]
    assert np.array_equal(gk.float().cpu().numpy(), wk) and np.array_equal(gv.float().cpu().numpy(), wv)


def test_read_without_tables_and_of_a_nan_scale(ss):
    """Page j = block j of a region of its own; a NaN scale reads as NaN."""
    rng = np.random.default_rng(32)
    blk = 16
    s = Stored(rng, blk, 0, [4 * blk], 2, 1).to_device()
    s.d_rec[1, 2, 2 * blk * D:2 * blk * D + 4] = torch.tensor([0, 0, 0xC0, 0x7F], dtype=torch.uint8)
    out = empty(4 * blk, 2, 2, D, fill=9.0, dtype=torch.bfloat16)
    ss.ss_read_kv8(s.d_rec, s.d_region, None, 0, s.n, s.d_open, s.d_len, dev([0, 4 * blk]), 1, 2, blk, D, 4 * blk, 0,
                   out.data_ptr(), out.data_ptr() + 2 * D, 2 * 4 * D, 4 * D)
    got = out.float().cpu().numpy()
    want = np.stack([ref.bf16(s.k[:, :4].astype(np.float32)), ref.bf16(s.v[:, :4].astype(np.float32))], 3)
    want = want.transpose(1, 2, 0, 3, 4).reshape(4 * blk, 2, 2, D)
    want[2 * blk:3 * blk, 1, 0] = np.nan
    assert np.array_equal(got, want, equal_nan=True)


# --------------------------------------------------------------- attention
@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("G, hkv", [(1, 5), (4, 2), (7, 1), (16, 2)])
def test_attention_over_selected_blocks(ss, blk, fmt, G, hkv):
    """Selections with holes, beyond the sequence, empty, twice the same, in
    any order, of one entry and of many (several splits)."""
    rng = np.random.default_rng(41 + blk + G)
    s = Stored(rng, blk, fmt, [0, 5, 3 * blk + 1, 40 * blk, 129 * blk + 7], hkv, G).to_device()
    for k in (1, 3, 37, 700):
        sel = rng.integers(-1, 140, (s.B, hkv, k)).astype(np.int32)
        sel[1], sel[3, 0] = -1, 2 ** 30
        sel[4, :, 0] = 128
        worst = s.check(attend(ss, s, sel), lambda b, g: sel[b, g], False)
        print(f"[gpu] k={k}: max abs error {worst:.2e}")


@pytest.mark.parametrize("blk", [8, 16, 32])
@pytest.mark.parametrize("fmt", [0, 1])
def test_attention_over_all_blocks_and_the_open_one(ss, blk, fmt):
    """Lengths from nothing to many blocks, every number of open tokens; what
    lies behind the last open token is not read into the result."""
    rng = np.random.default_rng(43)
    length = list(range(0, 2 * blk + 2)) + [17 * blk + 1, 300 * blk + blk - 1, 64 * blk]
    s = Stored(rng, blk, fmt, length, 2, 4)
    for b, n in enumerate(length):  # rows behind the last token
        s.open_k[b, :, n % blk:], s.open_v[b, :, n % blk:] = np.nan, np.inf
    s.to_device()
    for k in (301, 600, 16):
        out = attend(ss, s, None, k, with_open=True)
        s.check(out, lambda b, g: range(min(k, s.nblk[b])), True)


def test_attention_takes_any_workspace(ss):
    """None, too small for what the plan wants, and misaligned to 16 bytes."""
    rng = np.random.default_rng(44)
    s = Stored(rng, 16, 1, [900 * 16 + 3], 2, 7).to_device()
    one = 14 * 130 * 4
    full = ss.ss_sparse_attention_kv8_workspace(1, 14, 2, D, 16, 900)
    assert full > 4 * one
    for room in (0, one, 2 * one + 5, 3 * one, full, full + 999):
        out = attend(ss, s, None, 900, with_open=True, room=room)
        s.check(out, lambda b, g: range(900), True)


def test_attention_over_cache_slots(ss):
    """Slots of regions of different capacity: entries at or above a unit's own are skipped."""
    rng = np.random.default_rng(45)
    blk, hkv, B = 8, 2, 3
    s = Stored(rng, blk, 0, [64 * blk] * B, hkv, 4).to_device()
    cap = np.array([[7, 64], [0, 30], [64, 1]])
    region = np.zeros((B, hkv), np.int64)
    for b in range(B):  # unit (b, g) owns pages 60b .. of head g's records
        region[b] = (np.arange(hkv) * s.n + 60 * b) * ref.record_bytes(blk)
    sel = rng.integers(-1, 66, (B, hkv, 50)).astype(np.int32)
    out = host(attend(ss, s, sel, tables=False, nblk=False, capacity=dev(cap), limit=64, region=dev(region, np.int64)))
    for b in range(B):
        for g in range(hkv):
            pages = [60 * b + e for e in sel[b, g] if 0 <= e < cap[b, g]]
            k = s.k[g, pages].reshape(-1, D)
            v = s.v[g, pages].reshape(-1, D)
            want, bound = ref.attention(s.q[b, 4 * g:4 * g + 4].astype(np.float64), k, v, SCALE)
            assert (np.abs(out[b, 4 * g:4 * g + 4] - want) <= bound).all(), (b, g)


def test_attention_bad_pages_are_skipped(ss):
    """Tables with entries outside the pool, and blocks past the table's row."""
    rng = np.random.default_rng(46)
    s = Stored(rng, 16, 0, [20 * 16, 30 * 16], 1, 2)
    s.tables[0, 3], s.tables[0, 7], s.tables[1, 0] = s.n, -2, 2 ** 30
    s.to_device()
    s.check(attend(ss, s, None, 31), lambda b, g: range(31), False)
    s.max_blocks = 12
    s.d_tables = dev(s.tables[:, :12])
    s.tables = s.tables[:, :12]
    s.check(attend(ss, s, None, 31), lambda b, g: range(12), False)


def test_attention_past_4_gib(ss):
    """Pages and regions whose offsets pass 32 bits."""
    rng = np.random.default_rng(47)
    blk, rec = 16, ref.record_bytes(16)
    s = Stored(rng, blk, 0, [6 * blk, 6 * blk], 2, 4).to_device()
    high = (1 << 32) // rec + 5  # pages from here on lie past 4 GiB of a region
    big = torch.zeros(2 * (high + s.n) * rec, dtype=torch.uint8, device="cuda")
    view = big.view(2, high + s.n, rec)
    view[:, high:] = s.d_rec
    tables = np.where(s.tables >= 0, s.tables + high, -1)
    s.d_tables = dev(tables)
    region = dev(np.tile(np.arange(2) * (high + s.n) * rec, 2), np.int64)
    s.check(attend(ss, s, None, 7, rec=big, region=region, limit=high + s.n), lambda b, g: range(7), False)


@pytest.mark.parametrize("room", [0, None])
def test_attention_of_a_tile_that_is_not_finite(ss, room):
    """A NaN scale makes its unit's heads NaN, and no other's; unselected it
    does nothing.  Also where it is all that the unit attends."""
    rng = np.random.default_rng(48)
    s = Stored(rng, 16, 0, [200 * 16, 16], 2, 3)
    for page in (s.tables[0, 150], s.tables[1, 0]):
        s.rec[1, page, 2 * 16 * D:2 * 16 * D + 4] = np.array([np.nan], np.float32).view(np.uint8)
    s.rec[0, s.tables[0, 9], 2 * 16 * D + 4:2 * 16 * D + 8] = np.array([np.nan], np.float32).view(np.uint8)
    s.to_device()
    out = host(attend(ss, s, None, 200, room=room))
    nan = np.isnan(out)
    assert nan[0].all() and not nan[1, :3].any() and nan[1, 3:].all()
    sel = np.tile(np.arange(100, 149, dtype=np.int32), (2, 2, 1))
    s.check(attend(ss, s, sel, room=room), lambda b, g: sel[b, g], False)


@pytest.mark.parametrize("part", [0, 4])  # the K scale, the V scale
@pytest.mark.parametrize("every", [False, True])
def test_attention_keeps_a_nan_of_no_weight(ss, part, every):
    """A NaN tile far below the others' logits, in another wave and another
    split than theirs: its weight is 0 in fp32, its NaN stays."""
    rng = np.random.default_rng(53)
    B = 24 if every else 1
    s = Stored(rng, 16, 0, [1200 * 16] + [16] * (B - 1), 2, 4)
    s.q = ref.bf16(s.q * 0 + 300)  # a logit is the sum of a key's channels
    low = s.tables[0, 700]
    codes = s.rec[0, low, :16 * D]
    codes[:] = (codes & 0x7F) | 0x80  # negative keys: the lowest logits
    s.rec[0, low, 2 * 16 * D + part:2 * 16 * D + part + 4] = np.array([np.nan], np.float32).view(np.uint8)
    s.to_device()
    out = host(attend(ss, s, None, 1200, room=None))
    nan = np.isnan(out)
    assert nan[0, :4].all() and not nan[0, 4:].any() and not nan[1:].any()


def test_attention_large_logits(ss):
    """Logits in the thousands: the maximum is taken out before exp."""
    rng = np.random.default_rng(49)
    s = Stored(rng, 16, 1, [33 * 16], 1, 4)
    s.q = ref.bf16(s.q * 400)
    s.to_device()
    s.check(attend(ss, s, None, 33), lambda b, g: range(33), False)


def test_attention_of_queries_that_are_not_finite(ss):
    """A head whose query holds an infinity or a NaN is NaN, the others of its
    unit are not; where nothing is selected it is 0 all the same."""
    rng = np.random.default_rng(51)
    s = Stored(rng, 16, 0, [40 * 16 + 3, 16 * 5, 3], 2, 4)
    s.q[0, 1, 77], s.q[0, 6, 0], s.q[1, 0, 5], s.q[2, 3, 1] = np.nan, np.inf, -np.inf, np.nan
    s.to_device()
    sel = rng.integers(-1, 41, (3, 2, 30)).astype(np.int32)
    sel[1, 0] = -1  # nothing for the head with -inf
    for chosen, k, with_open in ((sel, None, False), (None, 41, True)):
        out = host(attend(ss, s, chosen, k, with_open=with_open))
        nan = np.isnan(out)
        want = np.zeros((3, 8), bool)
        want[0, [1, 6]] = True
        want[1, 0], want[2, 3] = chosen is None, chosen is None
        assert np.array_equal(nan, np.broadcast_to(want[:, :, None], nan.shape))
        if chosen is not None:
            assert (out[1, :4] == 0).all() and (out[2] == 0).all()


@pytest.mark.parametrize("fmt", [0, 1])
def test_attention_of_scales_far_apart(ss, fmt):
    """Tiles whose K and V scales differ by 2^24 within a unit, large ones
    first, last and between; queries with channels 2^-30 of their largest."""
    rng = np.random.default_rng(52)
    for order in (1, -1):
        s = Stored(rng, 16, fmt, [64 * 16, 64 * 16 + 9], 2, 4)
        grow = np.exp2(np.linspace(-12, 12, s.n))[::order]
        for g in range(2):
            for page in range(s.n):
                at = s.rec[g, page, 2 * 16 * D + 4:2 * 16 * D + 8].view(np.float32)
                at *= np.float32(grow[page] if g else grow[rng.integers(s.n)])
        s.q *= ref.bf16(np.exp2(rng.integers(-30, 1, s.q.shape)))
        s.k, s.v = ref.unpack(s.rec, 16, fmt)
        s.to_device()
        s.check(attend(ss, s, None, 64, with_open=True), lambda b, g: range(64), True)
        s.check(attend(ss, s, None, 64, with_open=True, room=0), lambda b, g: range(64), True)


def test_attention_of_infinite_open_values(ss):
    """An infinity in an open V row: not finite in that channel, the others as
    they are.  A probability enters in three bf16 parts, none negative: an
    infinity times a positive one is infinite, times 0 (the last part of a
    probability of 16 bits or fewer, such as 1) NaN."""
    rng = np.random.default_rng(54)
    s = Stored(rng, 16, 0, [5 * 16 + 7, 9], 2, 4)
    s.open_v[0, 1, 3, 50], s.open_v[1, 0, 8, 127] = np.inf, -np.inf
    s.to_device()
    out = host(attend(ss, s, None, 6, with_open=True))
    want = np.zeros(out.shape, bool)
    want[0, 4:, 50], want[1, :4, 127] = True, True
    assert np.array_equal(~np.isfinite(out), want)
    s.open_v[0, 1, 3, 50], s.open_v[1, 0, 8, 127] = 0, 0  # the other channels by the formula
    for b in range(2):
        for g in range(2):
            k, v = s.tokens(b, g, range(6), int(s.len[b]) % 16)
            heads = slice(4 * g, 4 * g + 4)
            plain, bound = ref.attention(s.q[b, heads].astype(np.float64), k, v, SCALE)
            assert ((np.abs(out[b, heads] - plain) <= bound) | want[b, heads]).all()


def test_two_streams_at_once(ss):
    """Calls that overlap, each with its own workspace: the results of calls alone."""
    rng = np.random.default_rng(55)
    sets = [Stored(rng, 16, 0, [3000 * 16 + 3, 70 * 16], 2, 4).to_device(), Stored(rng, 8, 1, [2500 * 8] * 14, 3, 4).to_device()]
    alone = [attend(ss, s, None, s.max_blocks, with_open=True) for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(6):
        for i, s in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                got[i].append(attend(ss, s, None, s.max_blocks, with_open=True))
    torch.cuda.synchronize()
    for want, results in zip(alone, got):
        assert all(torch.equal(want, r) for r in results)


def test_results_repeat_and_streams(ss):
    """The same bits again, and on another stream than the current one."""
    rng = np.random.default_rng(50)
    s = Stored(rng, 8, 1, [500 * 8 + 3, 70 * 8], 2, 7).to_device()
    first = attend(ss, s, None, 501, with_open=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (None, side):
        again = attend(ss, s, None, 501, with_open=True, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(first, again)


# ----------------------------------------------------- the calls together
class Serving:
    """A batch over a shared pool: the model holds every token's K and V."""

    def __init__(self, ss, rng, B, blk, fmt, hkv, G, max_blocks, n_pages, cap):
        self.ss, self.rng, self.B, self.blk, self.fmt, self.hkv, self.G, self.cap = ss, rng, B, blk, fmt, hkv, G, cap
        self.t = Tables(ss, B, blk, max_blocks, n_pages, rng)
        rec = ref.record_bytes(blk)
        self.records = torch.zeros(hkv, n_pages, rec, dtype=torch.uint8, device="cuda")
        self.region = dev(np.tile(np.arange(hkv) * n_pages * rec, B), np.int64)
        self.open = torch.zeros(B, hkv, 2 * blk * D, dtype=torch.bfloat16, device="cuda")
        self.meta = torch.zeros(B, hkv, max_blocks, 2, D, dtype=torch.bfloat16, device="cuda")
        self.k, self.v = [np.zeros((0, hkv, D), np.float32)] * B, [np.zeros((0, hkv, D), np.float32)] * B
        self.new = torch.zeros(cap, hkv, 2, D, dtype=torch.bfloat16, device="cuda")
        self.n_new = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.q = torch.zeros(B, hkv * G, D, dtype=torch.bfloat16, device="cuda")
        self.begin, self.taken, self.status = empty(B + 1), empty(B + 1), empty(B)
        self.slots, self.pos = empty(cap), empty(cap)
        self.topk = 4
        self.scores = torch.zeros(B, hkv, max_blocks, device="cuda")
        self.sel = empty(B, hkv, self.topk)
        self.out = torch.zeros(2, B, hkv * G, D, device="cuda")
        self.need = ss.ss_sparse_attention_kv8_workspace(B, hkv * G, hkv, D, blk, max_blocks)
        self.ws = empty(max(self.need, 16), fill=0xFF, dtype=torch.uint8)

    def feed(self, n_new):
        """The step's tokens and queries into the buffers that the calls read."""
        n = int(np.sum(n_new))
        k, v = values(self.rng, n, self.hkv, D), values(self.rng, n, self.hkv, D)
        self.new[:n] = to_bf16(np.stack([k, v], 2))
        self.n_new.copy_(dev(n_new))
        q = ref.bf16(self.rng.standard_normal((self.B, self.hkv * self.G, D)))
        self.q.copy_(to_bf16(q))
        self.host_q = q.astype(np.float64)
        at = 0
        for b in range(self.B):
            self.k[b] = np.concatenate([self.k[b], k[at:at + n_new[b]]])
            self.v[b] = np.concatenate([self.v[b], v[at:at + n_new[b]]])
            at += n_new[b]

    def step(self):
        """What a serving step enqueues: places, write, selection, both attentions."""
        ss, t, B, blk = self.ss, self.t, self.B, self.blk
        ss.ss_block_tables(t.len, self.n_new, t.n_free, B, blk, t.max_blocks, t.n_pages, t.free, t.tables, t.len, t.nblk,
                           t.n_free, self.begin, self.slots, self.pos, self.cap, self.taken, self.status)
        base = self.new.data_ptr()
        ss.ss_write_kv8(base, base + 2 * D, self.hkv * 4 * D, 4 * D, self.begin, self.slots, self.pos, B, self.hkv, blk,
                        D, self.cap, self.fmt, self.records, self.region, t.n_pages, self.open, self.meta, 0,
                        t.max_blocks)
        ss.ss_score_topk(self.q, self.meta, t.nblk, B, self.hkv * self.G, self.hkv, t.max_blocks, D, self.topk,
                         self.scores, self.sel)
        for i, sel in enumerate((self.sel, None)):
            ss.ss_sparse_attention_kv8(self.q, self.records, self.region, sel, t.tables, t.max_blocks, None, t.n_pages,
                                       t.nblk, self.open, t.len, self.fmt, B, self.hkv * self.G, self.hkv, D, blk,
                                       self.topk if sel is not None else t.max_blocks, SCALE, self.out[i], self.ws,
                                       self.need)

    def finish(self, done):
        self.t.release(done, check=False)
        for b in np.flatnonzero(done):
            self.k[b] = self.v[b] = self.k[b][:0]

    def check(self):
        """Both outputs from the model's tokens: quantised where their block is full."""
        torch.cuda.synchronize()
        blk = self.blk
        out, sel = host(self.out).astype(np.float64), host(self.sel)
        assert np.array_equal(host(self.t.len), [len(k) for k in self.k])
        assert (host(self.status) == 0).all()
        for b in range(self.B):
            full = len(self.k[b]) // blk
            tiles = [x[:full * blk].reshape(full, blk, self.hkv, D).transpose(2, 0, 1, 3) for x in (self.k[b], self.v[b])]
            if full:
                k, v = ref.unpack(ref.pack(*tiles, blk, self.fmt), blk, self.fmt)
            for g in range(self.hkv):
                chosen = sel[b, g][sel[b, g] >= 0]
                assert len(chosen) == min(full, self.topk)
                rest = [x[full * blk:, g].astype(np.float64) for x in (self.k[b], self.v[b])]
                heads = slice(g * self.G, (g + 1) * self.G)
                for i, blocks in enumerate((chosen, np.arange(full))):
                    kk = np.concatenate([k[g, blocks].reshape(-1, D), rest[0]]) if full else rest[0]
                    vv = np.concatenate([v[g, blocks].reshape(-1, D), rest[1]]) if full else rest[1]
                    want, bound = ref.attention(self.host_q[b, heads], kk, vv, SCALE)
                    assert (np.abs(out[i, b, heads] - want) <= bound).all(), (i, b, g)


@pytest.mark.parametrize("blk, fmt", [(8, 1), (16, 0), (32, 1)])
def test_serving_steps_over_a_shared_pool(ss, blk, fmt):
    """Prompts, decode steps, rows that finish and rows that join in their
    place, over a pool smaller than the rows' longest together."""
    rng = np.random.default_rng(61)
    B = 5
    s = Serving(ss, rng, B, blk, fmt, 2, 4, 24, 60, cap=400)
    steps = [[3 * blk + 5, 1, 0, 7 * blk, blk - 1], [1, 1, 1, 1, 1], [1] * 5, [0, 2 * blk + 1, 1, 1, 1], [1] * 5]
    done = [[0] * 5, [0, 0, 0, 1, 0], [0] * 5, [1, 1, 0, 0, 0], [0] * 5]
    for n_new, fin in zip(steps, done):
        s.feed(np.array(n_new))
        s.step()
        s.check()
        s.finish(np.array(fin))
    s.finish(np.ones(B))
    assert host(s.t.n_free)[0] == 60 and sorted(host(s.t.free)) == list(range(60))


def test_serving_step_in_a_graph(ss):
    """A decode step captured once and replayed as the sequences grow across
    block ends, with eager work and synchronisations between the replays;
    every replay is checked, and a second graph shares no buffer with it."""
    rng = np.random.default_rng(62)
    B, blk = 6, 8
    s = Serving(ss, rng, B, blk, 0, 2, 7, 20, 130, cap=B * 40)
    o = Serving(ss, rng, 3, 16, 1, 1, 4, 10, 40, cap=64)
    s.feed(np.array([37, 1, 8, 20, 7, 15]))
    s.step()
    s.check()
    o.feed(np.array([16, 3, 20]))
    o.step()
    o.check()
    graphs = []
    for x in (s, o):
        x.feed(np.ones(x.B, np.int64))  # a step of its own before the capture, which enqueues nothing
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            x.step()
        torch.cuda.current_stream().wait_stream(side)
        x.check()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.step()
        graphs.append(g)
    for i in range(10):
        n = np.ones(B, np.int64)
        n[i % B] = 0  # an idle row
        s.feed(n)
        o.feed(np.array([1, 0, 1]))
        graphs[0].replay()
        graphs[1].replay()
        s.check()
        o.check()
        if i == 4:
            s.finish(np.eye(1, B, 2)[0])


# ------------------------------------- equal shares of all sequences' steps
@pytest.mark.parametrize("blk, fmt, B, hkv, G, longest", [
    (8, 0, 14, 3, 4, 2100), (16, 1, 150, 2, 1, 300), (32, 0, 70, 1, 7, 200), (16, 0, 20, 2, 16, 400), (32, 1, 40, 1, 2, 20)])
def test_attention_of_long_tables_shared_out(ss, blk, fmt, B, hkv, G, longest):
    """Tables long enough that the workgroups share the steps of all
    sequences: lengths from nothing to `longest` blocks, so that shares begin
    and end inside units, span several, and units lie in one share or many."""
    rng = np.random.default_rng(71 + blk + B)
    length = (longest * blk * rng.random(B) ** 3).astype(int)
    length[rng.integers(B)] = longest * blk
    length[0] = 0
    k = max(longest, 700 * 32 // blk)
    s = Stored(rng, blk, fmt, length, hkv, G).to_device()
    first = attend(ss, s, None, k, with_open=True)
    worst = s.check(first, lambda b, g: range(s.nblk[b]), True)
    small = attend(ss, s, None, k, with_open=True, room=G * 130 * 4 * B * hkv)  # room for no share
    s.check(small, lambda b, g: range(s.nblk[b]), True)
    print(f"[gpu] max abs error {worst:.2e}")
    assert torch.equal(first, attend(ss, s, None, k, with_open=True))


# ------------------------------------------------- records in host memory
@pytest.mark.parametrize("blk", [8, 16, 32])
def test_gather_of_8_bit_records(ss, blk):
    """Missed records from mapped host memory into cache slots, byte for byte;
    rows out of range are skipped and other slots keep their bytes."""
    import ctypes
    rng = np.random.default_rng(81)
    rec, B, hkv, blocks, slots = ref.record_bytes(blk), 3, 2, 70, 9
    size = B * hkv * blocks * rec
    addr, mapped = ss.ss_host_alloc_mapped(size)
    pool = np.ctypeslib.as_array((ctypes.c_uint8 * size).from_address(addr)).reshape(B * hkv, blocks, rec)
    pool[:] = rng.integers(0, 256, pool.shape)
    cache = empty(B * hkv, slots, rec, fill=0x11, dtype=torch.uint8)
    want = np.full(cache.shape, 0x11, np.uint8)
    miss = [(b, g, int(rng.integers(blocks)), int(s)) for b in range(B) for g in range(hkv)
            for s in rng.permutation(slots)[:int(rng.integers(1, slots))]]
    for b, g, j, s in miss:
        want[b * hkv + g, s] = pool[b * hkv + g, j]
    bad = [(B, 0, 0, 0), (0, hkv, 0, 0), (0, 0, blocks, 0), (0, 0, 0, slots), (-1, 0, 0, 0), (0, 0, -1, 0)]
    rows = dev(miss[:5] + bad + miss[5:])
    off = lambda n: dev(np.arange(B * hkv) * n * rec, np.int64)  # noqa: E731
    ss.ss_gather_blocks(rows, len(rows), mapped, off(blocks), cache, off(slots), dev([blocks] * B),
                        dev([slots] * (B * hkv)), B, hkv, rec)
    got = host(cache)
    ss.ss_host_free(addr)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("blk, fmt", [(16, 0), (8, 1)])
def test_steps_over_a_hierarchical_cache_in_8_bits(ss, blk, fmt):
    """Prompts and single tokens written in 8 bits straight to the DRAM pool;
    each step scores, selects, resolves the slot tables, gathers the missing
    records and attends over the HBM cache's slots."""
    import ctypes
    rng = np.random.default_rng(82)
    rec, B, hkv, G, room, k, slots = ref.record_bytes(blk), 3, 2, 4, 40, 6, 9
    size = B * hkv * room * rec
    addr, mapped = ss.ss_host_alloc_mapped(size)
    pool = np.ctypeslib.as_array((ctypes.c_uint8 * size).from_address(addr))
    pool[:] = 0
    units = B * hkv
    pool_off, cache_off = (dev(np.arange(units) * n * rec, np.int64) for n in (room, slots))
    open_blocks = torch.zeros(B, hkv, 2 * blk * D, dtype=torch.bfloat16, device="cuda")
    meta = torch.zeros(B, hkv, room, 2, D, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(units, slots, rec, dtype=torch.uint8, device="cuda")
    capacity = np.full(units, slots, np.int32)
    handle = ss.ss_cache_create(B, hkv, np.zeros(B, np.int32), capacity, rec)
    keys, vals = [np.zeros((0, hkv, D), np.float32)] * B, [np.zeros((0, hkv, D), np.float32)] * B
    missed = 0
    try:
        for step, n_new in enumerate([[11 * blk + 3, 2 * blk - 1, 9 * blk], [1, 1, 1], [blk + 2, 1, 4 * blk], [1] * 3, [1] * 3]):
            n = sum(n_new)
            nk, nv = values(rng, n, hkv, D), values(rng, n, hkv, D)
            new = to_bf16(np.stack([nk, nv], 2))
            begin = np.concatenate([[0], np.cumsum(n_new)])
            pos = np.concatenate([len(keys[b]) + np.arange(n_new[b]) for b in range(B)])
            base = new.data_ptr()
            at = dev(pos)  # block j of a unit is record j of its region: slots are positions
            ss.ss_write_kv8(base, base + 2 * D, hkv * 4 * D, 4 * D, dev(begin), at, at, B, hkv, blk, D, n, fmt, mapped,
                            pool_off, room, open_blocks, meta, 0, room)
            for b in range(B):
                keys[b] = np.concatenate([keys[b], nk[begin[b]:begin[b + 1]]])
                vals[b] = np.concatenate([vals[b], nv[begin[b]:begin[b + 1]]])
            nblk = np.array([len(x) // blk for x in keys], np.int32)
            ss.ss_cache_set_blocks(handle, nblk)
            q = ref.bf16(rng.standard_normal((B, hkv * G, D)))
            d_q, d_nblk = to_bf16(q), dev(nblk)
            scores, sel = torch.zeros(B, hkv, room, device="cuda"), empty(B, hkv, k)
            ss.ss_score_topk(d_q, meta, d_nblk, B, hkv * G, hkv, room, D, k, scores, sel)
            sel = host(sel)
            slot, miss = np.zeros((B, hkv, k), np.int32), np.zeros((units * k, 4), np.int32)
            n_miss = ss.ss_cache_resolve(handle, step, sel, k, slot, miss, units * k)
            missed += n_miss
            ss.ss_gather_blocks(dev(miss), n_miss, mapped, pool_off, cache, cache_off, d_nblk, dev(capacity), B, hkv, rec)
            out = torch.zeros(B, hkv * G, D, device="cuda")
            d_len = dev([len(x) for x in keys])
            ss.ss_sparse_attention_kv8(d_q, cache, cache_off, dev(slot), None, 0, dev(capacity), slots, None, open_blocks,
                                       d_len, fmt, B, hkv * G, hkv, D, blk, k, SCALE, out, None, 0)
            out = host(out).astype(np.float64)
            for b in range(B):
                full = int(nblk[b])
                tiles = [x[:full * blk].reshape(full, blk, hkv, D).transpose(2, 0, 1, 3) for x in (keys[b], vals[b])]
                kk, vv = ref.unpack(ref.pack(*tiles, blk, fmt), blk, fmt)
                for g in range(hkv):
                    chosen = sel[b, g][sel[b, g] >= 0]
                    assert len(chosen) == min(full, k)
                    k_all = np.concatenate([kk[g, chosen].reshape(-1, D), keys[b][full * blk:, g].astype(np.float64)])
                    v_all = np.concatenate([vv[g, chosen].reshape(-1, D), vals[b][full * blk:, g].astype(np.float64)])
                    heads = slice(g * G, (g + 1) * G)
                    want, bound = ref.attention(q[b, heads].astype(np.float64), k_all, v_all, SCALE)
                    assert (np.abs(out[b, heads] - want) <= bound).all(), (step, b, g)
        assert 0 < missed < 5 * units * k
    finally:
        torch.cuda.synchronize()
        ss.ss_cache_destroy(handle)
        ss.ss_host_free(addr)
