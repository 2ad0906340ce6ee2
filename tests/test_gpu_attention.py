"""A block's attention on the GPU: rotation of the heads, attention over prompts, the 8-bit cache and attention over it, and a
run of them together with the block's linears, against plain forms in 64 bits (attention_reference)."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2508_04405_amd as fq
from gpu_helpers import say, to_dev

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")


def host(t):
    return t.cpu().numpy()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def starts_of(parts):
    return i32([0] + list(np.cumsum(parts)))


def normal(rng, *shape, size=1.0):
    return (size * rng.standard_normal(shape)).astype(np.float16)


def keys(rng, rows, width):
    """Some channels several times as large as the rest."""
    return (rng.standard_normal((rows, width)) * (1 + 4 * (rng.random(width) < 0.04))).astype(np.float16)


def assert_within(got, want, off, what=""):
    err = np.abs(got.astype(np.float64) - want)
    assert np.isfinite(got).all(), what
    assert (err <= off).all(), (what, float((err / off).max()), np.argwhere(err > off)[:4].tolist())


# ---- rotation --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("M,heads,kv,D,rot,interleaved,norm", [
    (1, 64, 8, 128, 128, False, False), (1, 1, 1, 64, 16, True, True), (3, 5, 5, 64, 64, False, True), (7, 24, 6, 64, 32, True, True),
    (33, 40, 40, 128, 32, False, True), (130, 6, 2, 128, 112, True, False), (2047, 4, 1, 64, 48, False, True),
    (2050, 8, 2, 128, 128, False, True), (2049, 3, 1, 64, 64, True, False), (1, 500, 12, 128, 128, False, True)])
def test_rotate(M, heads, kv, D, rot, interleaved, norm):
    say(f"rotate M={M} heads={heads}/{kv} D={D} rot={rot} interleaved={interleaved} norm={norm}")
    rng = np.random.default_rng([M, heads, D, rot])
    x = normal(rng, M, (heads + 2 * kv) * D + 8)
    positions = rng.integers(0, 1 << 20, M).astype(np.int32)
    positions[0] = 0
    freq = (10000.0 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    gq, gk = (normal(rng, D), normal(rng, D)) if norm else (None, None)
    want, off = ref.rotate(x, heads, kv, D, positions, freq, gq, gk, 1e-5, interleaved)
    kw = dict(gamma_q=None if gq is None else to_dev(gq), gamma_k=None if gk is None else to_dev(gk), interleaved=interleaved)
    dx, dp, df = to_dev(x), to_dev(positions), to_dev(freq)
    y = host(fq.rotate_heads(dx, heads, kv, D, dp, df, **kw))
    assert_within(y, want, off)
    width = (heads + kv) * D
    wide = torch.full((M, width + 24), 7.0, dtype=torch.float16, device=DEV)
    fq.rotate_heads(dx, heads, kv, D, dp, df, out=wide, **kw)
    assert np.array_equal(host(wide)[:, :width], y) and (host(wide)[:, width:] == 7.0).all()
    assert fq.rotate_heads(dx, heads, kv, D, dp, df, out=dx, **kw) is dx       # in place: the values' heads stay
    assert np.array_equal(host(dx)[:, :width], y) and np.array_equal(host(dx)[:, width:], x[:, width:])


def test_rotate_far_and_negative_positions_and_one_norm():
    rng = np.random.default_rng(5)
    positions = np.array([2**31 - 1, -2**31, -1, 0, 1, 123456789, -1000003, 31], np.int32)
    freq = np.array([1.0, 0.999, 3.0, 0.1, 1e-4, 1e-7, 0.5, 2.0], np.float32)
    x, g = normal(rng, 8, 4 * 64), normal(rng, 64)
    # 2^31 turns are counted with 53 bits: the angle is good to 2^-20 there
    want, off = ref.rotate(x, 2, 1, 64, positions, freq, gamma_k=g)
    y = host(fq.rotate_heads(to_dev(x), 2, 1, 64, to_dev(positions), to_dev(freq), gamma_k=to_dev(g)))
    assert_within(y, want, off + 2.0**-19 * np.abs(want).max())
    zero = host(fq.rotate_heads(to_dev(0 * x), 2, 1, 64, to_dev(positions), to_dev(freq), gamma_q=to_dev(g), gamma_k=to_dev(g)))
    assert not zero.any()


# ---- prompts ---------------------------------------------------------------------------------------------------

def check_prompt(q, k, v, parts, heads, kv, got, scale):
    at = 0
    for n in parts:
        if n:
            want, off = ref.grouped(q[at:at + n], k[at:at + n], v[at:at + n], heads, kv, 0, scale)
            assert_within(got[at:at + n], want, off, f"sequence at {at} of {n}")
        at += n


@pytest.mark.parametrize("heads,kv,D,parts", [
    (1, 1, 64, [1]), (1, 1, 128, [1]), (8, 1, 128, [1, 1, 1]), (4, 2, 64, [0, 5, 0, 0, 17, 1, 0]), (3, 1, 128, [63, 64, 65, 1, 129]),
    (5, 5, 64, [31, 33, 127, 128, 2]), (10, 2, 128, [300, 7, 211]), (2, 1, 64, [700]), (7, 1, 128, [260, 3]), (16, 1, 64, [90]),
    (80, 2, 64, [40, 11]), (2, 2, 128, [512, 257, 1, 1]), (4, 2, 128, [600]), (3, 1, 128, [515, 1000]), (6, 2, 64, [300, 212])])
def test_prompt(heads, kv, D, parts):
    say(f"prompt heads={heads}/{kv} D={D} {parts}")
    rng = np.random.default_rng([heads, D, sum(parts)])
    M, behind = sum(parts), 3
    fused = normal(rng, M + behind, (heads + 2 * kv) * D)
    fused[:, heads * D:(heads + kv) * D] = keys(rng, M + behind, kv * D)
    fused[M:] = NAN                                          # rows of no sequence
    f = to_dev(fused)
    q, k, v = f[:, :heads * D], f[:, heads * D:(heads + kv) * D], f[:, (heads + kv) * D:]
    out = torch.full((M + behind, heads * D + 8), 3.0, dtype=torch.float16, device=DEV)
    got = fq.prompt_attention(q, k, v, heads, kv, starts_of(parts), out=out[:, :heads * D])
    got = host(out)
    assert (got[M:] == 3.0).all() and (got[:, heads * D:] == 3.0).all()
    check_prompt(host(q), host(k), host(v), parts, heads, kv, got[:, :heads * D], D ** -0.5)
    again = host(fq.prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), heads, kv, starts_of(parts)))
    assert np.array_equal(again[:M], got[:M, :heads * D])


@pytest.mark.parametrize("size,scale", [(0.01, 1.0), (8.0, 1.0), (30.0, 0.5), (200.0, 0.088)])
def test_prompt_flat_and_peaked(size, scale):
    """Scores from nearly equal ones to ones that leave a single key, rising along the sequence, so that the maximum moves."""
    rng = np.random.default_rng(9)
    heads, kv, D, n = 4, 2, 64, 333
    q, k, v = normal(rng, n, heads * D), keys(rng, n, kv * D), normal(rng, n, kv * D)
    k = (k.astype(np.float32) * size * (1 + np.arange(n)[:, None] / n) / 8).astype(np.float16)
    got = host(fq.prompt_attention(to_dev(q), to_dev(k), to_dev(v), heads, kv, starts_of([n]), scale=scale))
    check_prompt(q, k, v, [n], heads, kv, got, scale)


def test_prompt_of_many_rows():
    """As many rows as take 256 to a workgroup; some of every sequence against the plain form."""
    rng = np.random.default_rng(10)
    heads, kv, D, parts = 64, 8, 128, [1500, 1, 2600, 7, 120, 31]
    M = sum(parts)
    q, k, v = normal(rng, M, heads * D), keys(rng, M, kv * D), normal(rng, M, kv * D)
    got = host(fq.prompt_attention(to_dev(q), to_dev(k), to_dev(v), heads, kv, starts_of(parts)))
    assert np.isfinite(got).all()
    at = 0
    for n in parts:
        for lo in sorted({0, n // 3, n // 2, max(n - 5, 0)}):
            hi = min(lo + 5, n)
            want, off = ref.grouped(q[at + lo:at + hi], k[at:at + hi], v[at:at + hi], heads, kv, lo, D ** -0.5)
            assert_within(got[at + lo:at + hi], want, off, f"rows {lo} .. {hi} of {n}")
        at += n


def test_prompt_of_the_smallest_scale():
    rng = np.random.default_rng(24)
    q, k, v = normal(rng, 70, 128), normal(rng, 70, 64), normal(rng, 70, 64)
    got = host(fq.prompt_attention(to_dev(q), to_dev(k), to_dev(v), 2, 1, starts_of([70]), scale=1.4e-45))
    check_prompt(q, k, v, [70], 2, 1, got, 1.4e-45)


@pytest.mark.parametrize("sign", [1, -1])
def test_prompt_of_the_largest_values(sign):
    """Weights whose rounding goes up: 512 and, from the second key on, 256.13, which fp16 takes for 256.25.  The mean of
    equal values is not beyond them."""
    n, D = 200, 64
    q, k, v = np.zeros((n, D), np.float16), np.zeros((n, D), np.float16), np.full((n, D), sign * 65504.0, np.float16)
    q[:, 0] = 1
    k[0, 0] = 1
    got = host(fq.prompt_attention(to_dev(q), to_dev(k), to_dev(v), 1, 1, starts_of([n]), scale=0.69265))
    check_prompt(q, k, v, [n], 1, 1, got, 0.69265)


def test_prompt_many_sequences():
    rng = np.random.default_rng(11)
    parts = rng.integers(0, 9, 700).tolist()
    heads, kv, D, M = 6, 3, 64, sum(parts)
    q, k, v = normal(rng, M, heads * D), keys(rng, M, kv * D), normal(rng, M, kv * D)
    got = host(fq.prompt_attention(to_dev(q), to_dev(k), to_dev(v), heads, kv, starts_of(parts)))
    check_prompt(q, k, v, parts, heads, kv, got, D ** -0.5)


# ---- the cache -------------------------------------------------------------------------------------------------

class Story:
    """Sequences that grow, in a cache and in plain rows beside it."""

    def __init__(self, rng, count, kv, D, page, most, extra_slots=0, scatter=True):
        per = -(-most // page)
        self.rng, self.kv, self.D, self.count = rng, kv, D, count
        pages = count * per + 3
        self.cache = fq.Cache(pages, page, kv, D, count + extra_slots)
        self.cache.codes.fill_(0xff)                         # (codes and, in the scales' place, NaN)
        self.cache.recent.fill_(0xff)
        order = rng.permutation(pages) if scatter else np.arange(pages)
        self.table = order[:count * per].reshape(count, per).astype(np.int32)
        self.slots = rng.permutation(count + extra_slots)[:count].astype(np.int32)
        self.k = [np.zeros((0, kv * D), np.float16) for _ in range(count)]
        self.v = [np.zeros((0, kv * D), np.float16) for _ in range(count)]

    def lengths(self):
        return [len(x) for x in self.k]

    def seqs(self, parts):
        return fq.Sequences(starts_of(parts), i32(self.lengths()), to_dev(self.table), to_dev(self.slots))

    def append(self, parts, make=None):
        M, width = sum(parts), self.kv * self.D
        k, v = make(M, width) if make else (keys(self.rng, M, width), normal(self.rng, M, width))
        at = 0
        for i, n in enumerate(parts):
            self.k[i] = np.concatenate([self.k[i], k[at:at + n]])
            self.v[i] = np.concatenate([self.v[i], v[at:at + n]])
            at += n
        if M:
            wide = np.full((M + 2, 2 * width + 16), NAN, np.float16)
            wide[:M, :width], wide[:M, width:2 * width] = k, v
            w = to_dev(wide)
            fq.cache_append(self.cache, w[:, :width], w[:, width:2 * width], self.seqs(parts))

    def cut(self, i, length):
        self.k[i], self.v[i] = self.k[i][:length], self.v[i][:length]

    def check_read(self, parts):
        M, width = sum(parts), self.kv * self.D
        out = torch.full((M + 2, 2 * width + 8), 5.0, dtype=torch.float16, device=DEV)
        fq.cache_read(self.cache, self.seqs(parts), out=(out[:, :width], out[:, width:2 * width]))
        got, at = host(out), 0
        assert (got[M:] == 5.0).all() and (got[:, 2 * width:] == 5.0).all()
        for i, n in enumerate(parts):
            for rows, part in ((self.k[i], got[at:at + n, :width]), (self.v[i], got[at:at + n, width:2 * width])):
                assert np.array_equal(part, ref.stored_half(rows, self.kv)[len(rows) - n:]), (i, n, len(rows))
            at += n

    def check_attention(self, parts, heads, scale=None, size=1.0):
        M, D = sum(parts), self.D
        q = normal(self.rng, M, heads * D, size=size)
        out = torch.full((M + 2, heads * D), 5.0, dtype=torch.float16, device=DEV)
        rows = to_dev(np.concatenate([q, np.full((2, heads * D), NAN, np.float16)]))
        fq.cache_attention(self.cache, rows, heads, self.seqs(parts), scale=scale, out=out)
        got, at = host(out), 0
        assert (got[M:] == 5.0).all()
        for i, n in enumerate(parts):
            L = len(self.k[i])
            want, off = ref.grouped(q[at:at + n], ref.stored(self.k[i], self.kv), ref.stored(self.v[i], self.kv), heads, self.kv,
                                    L - n, D ** -0.5 if scale is None else scale)
            assert_within(got[at:at + n], want, off, f"sequence {i} of {L}, {n} new")
            at += n
        return got


@pytest.mark.parametrize("kv,D,page", [(1, 64, 16), (2, 128, 16), (3, 64, 64), (2, 128, 128), (1, 128, 1024), (5, 64, 32)])
def test_cache_holds_what_it_should(kv, D, page):
    """Appends of every size, from every place in a block: each value is the codes' of its block once, whichever way it came."""
    say(f"cache kv={kv} D={D} page={page}")
    s = Story(np.random.default_rng([kv, D, page]), 5, kv, D, page, 300, extra_slots=2)
    for parts in ([1, 16, 15, 0, 200], [1, 1, 1, 1, 1], [14, 15, 17, 30, 33], [1, 0, 0, 2, 31], [16, 1, 32, 3, 7], [40, 60, 5, 33, 0]):
        s.append(parts)
        s.check_read(parts)
        s.check_read(s.lengths())
    s.check_read([0, 3, 20, 1, 90])


def test_cache_codes_are_the_activation_quantizers():
    rng = np.random.default_rng(2)
    s = Story(rng, 1, 2, 128, 16, 64)
    s.append([48])
    got_k, got_v = (host(t) for t in fq.cache_read(s.cache, s.seqs([48]), rows=48))
    for rows, got in ((s.k[0], got_k), (s.v[0], got_v)):
        flat = rows.reshape(3, 16, 2, 128).transpose(0, 2, 1, 3).reshape(6, 16 * 128)
        codes, scales = fq.quant_act(to_dev(flat), 8)
        want = (host(codes).astype(np.float32) * host(scales).astype(np.float32)[:, None]).astype(np.float16)
        assert np.array_equal(got, want.reshape(3, 2, 16, 128).transpose(0, 2, 1, 3).reshape(48, 256))


def test_cache_of_zeros_large_and_tiny_values():
    rng = np.random.default_rng(3)
    for what in (0.0, 65504.0, 6e-8, 1e-4):
        s = Story(rng, 2, 1, 64, 16, 80)
        make = lambda M, w: tuple((what * np.sign(rng.standard_normal((M, w)))).astype(np.float16) for _ in range(2))
        s.append([37, 64], make)
        s.check_read([37, 64])
        s.check_attention([3, 1], 4, scale=0.125 if what < 1 else 1e-9)


def test_a_sequence_can_be_shortened():
    """Back to the beginning of the block before the unfinished one, and on from there."""
    rng = np.random.default_rng(4)
    for L in (16, 17, 31, 32, 40, 47, 95):
        for back in range(max(0, 16 * (L // 16) - 16), L):
            s = Story(rng, 2, 1, 64, 16, 160)
            s.append([L // 2, 5])
            s.append([L - L // 2, 0])
            s.cut(0, back)
            if back:
                s.check_read([back, 5])
                s.check_attention([1, 1], 2)
            s.append([9, 30])
            s.check_read([back + 9, 35])
            s.append([30, 1])
            s.check_read([back + 39, 36])


@pytest.mark.parametrize("heads,kv,D,page,lengths,new", [
    (1, 1, 128, 16, [1], [1]), (8, 1, 128, 16, [16], [1]), (64, 8, 128, 64, [1100], [1]), (32, 32, 128, 16, [77], [1]),
    (8, 2, 64, 32, [1, 15, 16, 17, 31, 32, 33, 300], [1] * 8), (40, 8, 128, 128, [129, 3, 700], [1, 1, 1]),
    (24, 6, 64, 16, [50, 60, 400, 5], [4, 0, 8, 5]), (5, 1, 128, 32, [900, 200, 64], [3, 7, 64]),
    (16, 2, 64, 64, [333, 1000], [100, 300]), (16, 1, 128, 16, [2100], [130]), (34, 2, 128, 16, [40, 500], [1, 1]),
    (3, 3, 64, 1024, [3000, 2049], [1, 2]), (200, 1, 64, 16, [150], [1]), (12, 3, 64, 32, [400, 77, 150], [9, 12, 10]), (12, 3, 128, 32, [400, 77, 150], [9, 12, 10]), (70, 1, 128, 32, [90, 33], [1, 0])])
def test_cached_attention(heads, kv, D, page, lengths, new):
    say(f"cached heads={heads}/{kv} D={D} page={page} {lengths} {new}")
    rng = np.random.default_rng([heads, D, page, sum(lengths)])
    s = Story(rng, len(lengths), kv, D, page, max(lengths) + 5, extra_slots=1)
    s.append([n - m for n, m in zip(lengths, new)])
    s.append(new)
    s.check_attention(new, heads)
    s.check_attention(new, heads, scale=1.0, size=3.0)


def test_cached_attention_of_many_sequences():
    rng = np.random.default_rng(12)
    lengths = rng.integers(1, 40, 150)
    s = Story(rng, 150, 2, 64, 16, 48)
    s.append(lengths.tolist())
    s.check_attention([1] * 150, 8)
    s.check_attention(rng.integers(0, lengths + 1).tolist(), 8)


@pytest.mark.parametrize("heads,kv,D,count,most,new", [
    (32, 16, 64, 60, 500, 2), (16, 16, 128, 100, 200, 1), (40, 20, 128, 33, 90, 9), (64, 32, 64, 5, 40, 6), (12, 12, 64, 200, 64, 3),
    (4, 1, 64, 70, 900, 1), (16, 8, 64, 300, 20, 1)])
def test_many_sequences_of_any_length(heads, kv, D, count, most, new):
    """Many tiles of few steps each, and of more; some without tokens or rows."""
    rng = np.random.default_rng([26, D, count])
    lengths = rng.integers(0, most + 1, count)
    lengths[:3] = most, 0, 16
    rows = np.minimum(lengths, new)
    rows[3] = 0
    s = Story(rng, count, kv, D, 16, most)
    s.append((lengths - rows).tolist())
    s.append(rows.tolist())
    s.check_attention(rows.tolist(), heads)


@pytest.mark.parametrize("heads,kv,D", [(8, 2, 64), (4, 2, 128), (24, 1, 128)])
def test_long_sequences_with_holes(heads, kv, D):
    """Pages in the middle that are not there, and no slot, where several workgroups share a tile."""
    rng = np.random.default_rng([27, D])
    s = Story(rng, 3, kv, D, 32, 2100)
    s.append([2075, 1300, 1000])
    s.append([2, 0, 1])
    parts, q = (2, 0, 1), normal(rng, 3, heads * D)
    table = s.table.copy()
    table[0, 5:9], table[0, 40], table[2, 0] = -1, 2**30, -2**31
    out = host(fq.cache_attention(s.cache, to_dev(q), heads, fq.Sequences(starts_of(parts), i32(s.lengths()), to_dev(table),
                                                                        i32([s.slots[0], 0, -1]))))
    for rows, i, left, first in ((slice(0, 2), 0, np.r_[0:160, 288:1280, 1312:2077], 2075 - 160), (slice(2, 3), 2, np.r_[32:992], 960)):
        k, v = ref.stored(s.k[i], kv)[left], ref.stored(s.v[i], kv)[left]
        want, off = ref.grouped(q[rows], k, v, heads, kv, first, D ** -0.5)
        assert_within(out[rows], want, off, f"sequence {i}")


@pytest.mark.parametrize("heads,kv,D", [(8, 1, 64), (16, 2, 128)])
def test_chunks_of_many_sequences(heads, kv, D):
    """More than 64 rows of a sequence on average, of more than 64 sequences, some without rows, some without tokens."""
    rng = np.random.default_rng([19, D])
    count = 70
    new = rng.integers(0, 40, count)
    new[:4] = 0, 200, 1, 0
    before = rng.integers(0, 150, count)
    before[3] = 0
    s = Story(rng, count, kv, D, 32, 352)
    s.append(before.tolist())
    s.append(new.tolist())
    assert new.sum() * (heads // kv) / count > 64
    s.check_attention(new.tolist(), heads)


@pytest.mark.parametrize("D", [64, 128])
def test_chunks_that_see_nothing_or_not_all(D):
    rng = np.random.default_rng([20, D])
    kv, heads = 1, 8
    s = Story(rng, 3, kv, D, 16, 128)
    s.append([60, 80, 90])
    s.append([40, 30, 10])
    parts = (40, 30, 10)
    q = normal(rng, 80, heads * D)
    k, v = [ref.stored(x, kv) for x in s.k], [ref.stored(x, kv) for x in s.v]

    def run(lengths=(100, 110, 100), table=s.table, slots=s.slots, scale=None):
        seqs = fq.Sequences(starts_of(parts), i32(list(lengths)), to_dev(np.ascontiguousarray(table)), to_dev(slots))
        return host(fq.cache_attention(s.cache, to_dev(q), heads, seqs, scale=scale))

    def check(out, rows, k, v, first, scale=D ** -0.5):
        want, off = ref.grouped(q[rows], k, v, heads, kv, first, scale)
        assert_within(out[rows], want, off)

    # lengths below the rows: the first ones see nothing
    out = run(lengths=(16, 0, -3))
    assert not out[:24].any() and not out[40:].any()
    check(out, slice(24, 40), k[0][:16], v[0][:16], 0)
    # pages that are not there, the last one, which the unfinished block would go to, among them
    table = s.table.copy()
    table[0, 1], table[0, 6], table[1, :] = -1, 2**30, 2**31 - 1
    out = run(table=table)
    left = np.r_[0:16, 32:100]
    check(out, slice(0, 40), k[0][left], v[0][left], 44)
    # (the second sequence's pages: none; its unfinished block begins at 96, and its rows at 80)
    assert not out[40:56].any()
    check(out, slice(56, 70), k[1][96:], v[1][96:], 0)
    # slots that are not there
    out = run(slots=np.array([-1, 3, -2**31], np.int32))
    for rows, i, first in ((slice(0, 40), 0, 60), (slice(40, 70), 1, 80), (slice(70, 80), 2, 90)):
        check(out, rows, k[i][:96], v[i][:96], first)
    # the smallest scale, which a small scale of keys would take to zero
    out = run(scale=1.4e-45)
    for rows, i, first in ((slice(0, 40), 0, 60), (slice(40, 70), 1, 80), (slice(70, 80), 2, 90)):
        check(out, rows, k[i], v[i], first, 1.4e-45)


def test_starts_that_fall_or_lie_outside():
    """What they do not describe is left out or wrong; what they describe is right, and rows outside stay as they were."""
    rng = np.random.default_rng(25)
    kv, D, heads, M = 2, 64, 16, 100
    q, k, v = normal(rng, M, heads * D), keys(rng, M, kv * D), normal(rng, M, kv * D)
    s = Story(rng, 3, kv, D, 16, 160)
    s.append([30, 40, 50])
    for starts in ([0, 50, 20, 500], [-7, 10, 10, 60], [60, 60, 2**31 - 1, 3], [0, -2**31, 70, 90]):
        say(f"starts {starts}")
        out = torch.full((M + 8, heads * D), 5.0, dtype=torch.float16, device=DEV)
        fq.prompt_attention(to_dev(q), to_dev(k), to_dev(v), heads, kv, i32(starts), out=out[:M])
        got = host(out)
        assert np.isfinite(got).all() and (got[M:] == 5.0).all()
        if starts[0] == -7:
            for lo, hi in ((0, 10), (10, 60)):
                check_prompt(q[lo:hi], k[lo:hi], v[lo:hi], [hi - lo], heads, kv, got[lo:hi], D ** -0.5)
            assert (got[60:] == 5.0).all()
        seqs = fq.Sequences(i32(starts), i32(s.lengths()), to_dev(s.table), to_dev(s.slots))
        out.fill_(5.0)
        fq.cache_attention(s.cache, to_dev(q), heads, seqs, out=out[:M])
        got = host(out)
        assert np.isfinite(got).all() and (got[M:] == 5.0).all()
        back = torch.full((2, M + 8, kv * D), 5.0, dtype=torch.float16, device=DEV)
        fq.cache_read(s.cache, seqs, out=(back[0, :M], back[1, :M]))
        assert (host(back)[:, M:] == 5.0).all()
        pages = torch.full_like(s.cache.codes, 7)
        copy = fq.Cache(*s.cache.codes.shape[:1], 16, kv, D, s.cache.slots)
        copy.codes.copy_(pages)
        fq.cache_append(copy, to_dev(k), to_dev(v), seqs)
        unused = sorted(set(range(pages.shape[0])) - set(s.table.ravel().tolist()))
        assert torch.equal(copy.codes[unused], pages[unused])


def test_a_length_beyond_the_table_counts_as_its_end():
    rng = np.random.default_rng(21)
    s = Story(rng, 2, 1, 64, 16, 64)
    s.append([64, 20])
    q = to_dev(normal(rng, 4, 4 * 64))
    call = lambda first: host(fq.cache_attention(s.cache, q, 4, fq.Sequences(i32([0, 2, 4]), i32([first, 20]), to_dev(s.table),
                                                                           to_dev(s.slots))))
    want = call(64)
    for length in (65, 1000, 2**31 - 1):
        assert np.array_equal(call(length), want)


@pytest.mark.parametrize("n", [1, 12, 40])
def test_sequences_that_share_pages(n):
    """A beginning that two sequences have in common, in the same pages; tokens of their own behind it."""
    rng = np.random.default_rng([22, n])
    kv, D, heads, page = 2, 128, 4, 32
    s = Story(rng, 2, kv, D, page, 256)
    s.append([128, 0])
    s.table[1, :4] = s.table[0, :4]
    s.k[1], s.v[1] = s.k[0].copy(), s.v[0].copy()
    s.append([n, n])
    s.check_read(s.lengths())
    s.check_attention([n, n], heads)


def test_values_of_very_different_sizes():
    """Blocks whose values' scales are 2^20 apart."""
    rng = np.random.default_rng(13)

    def make(M, w):
        size = np.where(np.arange(M) // 16 % 3 == 0, 3e4, np.where(np.arange(M) // 16 % 3 == 1, 1.0, 3e-3))[:, None]
        return keys(rng, M, w), np.clip(rng.standard_normal((M, w)) * size, -6e4, 6e4).astype(np.float16)

    s = Story(rng, 2, 2, 64, 32, 400)
    s.append([390, 120], make)
    s.check_attention([2, 1], 4)


def test_a_row_that_sees_nothing():
    """Lengths below the rows of the batch, empty sequences, pages and slots that are not there."""
    rng = np.random.default_rng(14)
    kv, D, heads, page = 2, 64, 4, 16
    s = Story(rng, 3, kv, D, page, 64)
    s.append([40, 20, 33])
    good = s.check_attention([1, 1, 1], heads)
    assert np.isfinite(good[:3]).all()
    q = to_dev(normal(rng, 6, heads * D))
    seqs = lambda lengths, table=s.table, slots=s.slots, parts=(2, 2, 2): fq.Sequences(
        starts_of(parts), i32(lengths), to_dev(np.ascontiguousarray(table)), to_dev(slots))
    out = host(fq.cache_attention(s.cache, q, heads, seqs([40, 1, 0])))
    assert out[:2].any(1).all() and not out[2].any() and out[3].any() and not out[4:].any()
    read = [host(t) for t in fq.cache_read(s.cache, seqs([40, 1, -5]), rows=6)]
    for t in read:
        assert not t[2].any() and t[3].any() and not t[4:].any()
    # a page that is not there: its keys are not seen, by whole blocks
    table = s.table.copy()
    table[0, 1] = -1
    table[1, 0] = 2**30
    table[2, :] = -7
    bad = seqs([40, 20, 33], table)
    out = host(fq.cache_attention(s.cache, q, heads, bad))
    k, v = ref.stored(s.k[0], kv), ref.stored(s.v[0], kv)
    left = np.r_[0:16, 32:40]
    want, off = ref.grouped(host(q)[1:2], k[left], v[left], heads, kv, 23, D ** -0.5)
    assert_within(out[1:2], want, off)
    k, v = ref.stored(s.k[1], kv)[16:], ref.stored(s.v[1], kv)[16:]
    want, off = ref.grouped(host(q)[2:4], k, v, heads, kv, 2, D ** -0.5)
    assert_within(out[2:4], want, off)
    read = [host(t) for t in fq.cache_read(s.cache, seqs([40, 20, 33], table, parts=(40, 20, 33)), rows=93)]
    assert not read[0][16:32].any() and np.array_equal(read[0][32:40], ref.stored_half(s.k[0], kv)[32:])
    assert not read[1][40:56].any() and np.array_equal(read[1][56:60], s.v[1][16:])
    # slots that are not there: the unfinished block's tokens are not seen; nothing is written for them
    before = s.cache.codes.clone(), s.cache.recent.clone()
    slots = np.array([-1, 3, 2**31 - 1], np.int32)
    out = host(fq.cache_attention(s.cache, q, heads, seqs([40, 16, 33], slots=slots)))
    want, off = ref.grouped(host(q)[0:2], ref.stored(s.k[0], kv)[:32], ref.stored(s.v[0], kv)[:32], heads, kv, 32, D ** -0.5)
    assert_within(out[0:2], want, off)
    rows = to_dev(normal(rng, 6, kv * D))
    fq.cache_append(s.cache, rows, rows, seqs([42, 22, 35], table=-np.ones_like(s.table), slots=slots))
    assert torch.equal(s.cache.codes, before[0]) and torch.equal(s.cache.recent, before[1])


# ---- streams, graphs, large addresses --------------------------------------------------------------------------

def test_a_captured_step_follows_lengths_and_pages():
    """Append and attention in a graph, replayed while the sequences grow, with eager work between the replays."""
    rng = np.random.default_rng(15)
    kv, D, heads, count = 2, 128, 8, 3
    s = Story(rng, count, kv, D, 16, 400)
    s.append([30, 200, 1])
    k, v, q = (torch.zeros((count, w * D), dtype=torch.float16, device=DEV) for w in (kv, kv, heads))
    seqs = s.seqs([1, 1, 1])
    ws = torch.empty(fq.load().flexq_cache_attention_workspace_bytes(count, count, heads, kv, D), dtype=torch.uint8, device=DEV)
    out = torch.empty((count, heads * D), dtype=torch.float16, device=DEV)
    kk, vv = to_dev(normal(rng, 3, kv * D)), to_dev(normal(rng, 3, kv * D))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.cache_append(s.cache, k, v, seqs)
        fq.cache_attention(s.cache, q, heads, seqs, workspace=ws, out=out)
    for step in range(20):
        rows = keys(rng, count, kv * D), normal(rng, count, kv * D)
        for i in range(count):
            s.k[i] = np.concatenate([s.k[i], rows[0][i:i + 1]])
            s.v[i] = np.concatenate([s.v[i], rows[1][i:i + 1]])
        k.copy_(to_dev(rows[0]))
        v.copy_(to_dev(rows[1]))
        qh = normal(rng, count, heads * D)
        q.copy_(to_dev(qh))
        seqs.lengths.copy_(i32(s.lengths()))
        ws.fill_(step * 37 % 256)
        out.fill_(NAN)
        graph.replay()
        got = host(out)
        eager = host(fq.cache_attention(s.cache, q, heads, seqs))
        assert np.array_equal(got, eager)
        for i in range(count):
            want, off = ref.grouped(qh[i:i + 1], ref.stored(s.k[i], kv), ref.stored(s.v[i], kv), heads, kv, len(s.k[i]) - 1, D ** -0.5)
            assert_within(got[i:i + 1], want, off, f"step {step} sequence {i}")
    del kk, vv


@pytest.mark.parametrize("heads,kv,new", [(8, 2, 1), (8, 2, 6), (32, 16, 1), (8, 1, 20)])
def test_a_captured_call_meets_other_lengths(heads, kv, new):
    """Lengths, pages and slots that change between replays by so much that work is cut in another way."""
    rng = np.random.default_rng([28, kv, new])
    D, count = 64, 3
    s = Story(rng, count, kv, D, 32, 2100)
    s.append([2080, 1536, 2000])
    table, slots = to_dev(s.table), to_dev(s.slots)
    seqs = fq.Sequences(starts_of([new] * count), i32([32] * count), table, slots)
    q = torch.zeros((count * new, heads * D), dtype=torch.float16, device=DEV)
    out = torch.empty_like(q)
    ws = torch.empty(fq.load().flexq_cache_attention_workspace_bytes(count * new, count, heads, kv, D), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.cache_attention(s.cache, q, heads, seqs, workspace=ws, out=out)
    for lengths in ([32, 48, 32], [2080, 1536, 2000], [0, 1536, 32], [32, 32, 32], [512, 512, 512], [2080, 32, 48]):
        qh = normal(rng, count * new, heads * D)
        q.copy_(to_dev(qh))
        seqs.lengths.copy_(i32(lengths))
        ws.fill_(255)
        out.fill_(NAN)
        graph.replay()
        got = host(out)
        assert np.array_equal(got, host(fq.cache_attention(s.cache, q, heads, seqs)))
        for i, L in enumerate(lengths):
            rows = slice(i * new, (i + 1) * new)
            want, off = ref.grouped(qh[rows], ref.stored(s.k[i], kv)[:L], ref.stored(s.v[i], kv)[:L], heads, kv, L - new, D ** -0.5)
            assert_within(got[rows], want, off, f"lengths {lengths} sequence {i}")


def test_two_graphs_share_a_workspace():
    """Chunks of two sequences' prompts and single tokens, in graphs of one workspace, replayed in turn with eager calls and a
    changed batch between them."""
    rng = np.random.default_rng(23)
    kv, D, heads = 1, 64, 8
    s = Story(rng, 2, kv, D, 32, 700)
    s.append([600, 333])
    shapes = [[30, 25], [1, 1]]
    seqs = [s.seqs(parts) for parts in shapes]
    q = [torch.zeros((sum(parts), heads * D), dtype=torch.float16, device=DEV) for parts in shapes]
    k = [torch.zeros((sum(parts), kv * D), dtype=torch.float16, device=DEV) for parts in shapes]
    out = [torch.empty_like(x) for x in q]
    own = [torch.empty_like(x) for x in q]
    need = max(fq.load().flexq_cache_attention_workspace_bytes(sum(p), 2, heads, kv, D) for p in shapes)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in shapes]
    for i, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            fq.cache_attention(s.cache, q[i], heads, seqs[i], workspace=ws, out=out[i])
            fq.prompt_attention(q[i], k[i], k[i], heads, kv, seqs[i].starts, out=own[i])
    for step in range(5):
        for i, graph in enumerate(graphs):
            q[i].copy_(to_dev(normal(rng, *q[i].shape)))
            k[i].copy_(to_dev(normal(rng, *k[i].shape)))
            seqs[i].lengths.copy_(i32([600 - 37 * step, 333 - 16 * step]))
            out[i].fill_(NAN)
            own[i].fill_(NAN)
            graph.replay()
            got, got_own = host(out[i]), host(own[i])
            ws.fill_(255)
            assert np.array_equal(got, host(fq.cache_attention(s.cache, q[i], heads, seqs[i])))
            assert np.array_equal(got_own, host(fq.prompt_attention(q[i], k[i], k[i], heads, kv, seqs[i].starts)))
            assert np.isfinite(got).all() and np.isfinite(got_own).all()


def test_two_streams_at_once():
    rng = np.random.default_rng(16)
    kv, D, heads = 4, 128, 16
    stories = [Story(rng, 4, kv, D, 32, 600) for _ in range(2)]
    for s in stories:
        s.append([500, 3, 90, 310])
    q = [to_dev(normal(rng, 4, heads * D)) for _ in stories]
    seqs = [s.seqs([1, 1, 1, 1]) for s in stories]
    p = [to_dev(normal(rng, 200, heads * D)) for _ in stories]
    want = [host(fq.cache_attention(s.cache, x, heads, e)) for s, x, e in zip(stories, q, seqs)]
    want_p = [host(fq.prompt_attention(x, x[:, :kv * D], x[:, kv * D:2 * kv * D], heads, kv, starts_of([150, 50]))) for x in p]
    streams, got = [torch.cuda.Stream() for _ in stories], [[], []]
    st = starts_of([150, 50])
    torch.cuda.synchronize()
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append((fq.cache_attention(stories[i].cache, q[i], heads, seqs[i]),
                               fq.prompt_attention(p[i], p[i][:, :kv * D], p[i][:, kv * D:2 * kv * D], heads, kv, st)))
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in got[i]:
            assert np.array_equal(host(a), want[i]) and np.array_equal(host(b), want_p[i])


def test_a_cache_past_32_bits():
    """Pages and slots whose bytes, and rows whose elements, lie past 4 Gi."""
    rng = np.random.default_rng(17)
    kv, D, heads, page = 8, 128, 8, 1024
    per_page = fq.load().flexq_cache_page_bytes(kv, D, page)
    pages = (5 << 30) // per_page
    slots = (5 << 30) // fq.load().flexq_cache_recent_bytes(kv, D)
    cache = fq.Cache(pages, page, kv, D, slots)
    table, where = i32([[pages - 1, 0, pages - 2]]), i32([slots - 1])
    k, v = keys(rng, 2060, kv * D), normal(rng, 2060, kv * D)
    q = normal(rng, 3, heads * D)
    fq.cache_append(cache, to_dev(k), to_dev(v), fq.Sequences(i32([0, 2060]), i32([2060]), table, where))
    big = torch.empty((66000, 65536), dtype=torch.float16, device=DEV)        # 8.6 GB of rows
    rows = big[65990:65993, 65536 - heads * D:]
    rows.copy_(to_dev(q))
    got = host(fq.cache_attention(cache, rows, heads, fq.Sequences(i32([0, 3]), i32([2060]), table, where)))
    want, off = ref.grouped(q, ref.stored(k, kv), ref.stored(v, kv), heads, kv, 2057, D ** -0.5)
    assert_within(got, want, off)
    # prompts and rotation of rows far into such a buffer, as parts of one call: sequences at its two ends
    n, at = 70, 65800
    tail = big[at:at + n]
    big[:n, :3 * D].copy_(to_dev(normal(rng, n, 3 * D)))
    tail[:, :3 * D].copy_(to_dev(normal(rng, n, 3 * D)))
    starts = i32([0, n, n, at, at + n])
    view = big[:, :3 * D]
    view[n:at].zero_()
    out = big[:, 4 * D:5 * D]
    parts = view[:, :D], view[:, D:2 * D], view[:, 2 * D:]
    fq.prompt_attention(*parts, 1, 1, i32([0, n]), out=out)
    fq.prompt_attention(*(x[at:at + n] for x in parts), 1, 1, i32([0, n]), out=out[at:at + n])
    for lo in (0, at):
        h = host(view[lo:lo + n])
        want, off = ref.grouped(h[:, :D], h[:, D:2 * D], h[:, 2 * D:], 1, 1, 0, D ** -0.5)
        assert_within(host(out[lo:lo + n]), want, off)
    out.fill_(0)
    packed = i32([0, n] + [at] * 2 + [at + n])
    ends = i32([0] + [n + (at - n) * i // 64 for i in range(65)] + [at + n])      # the middle in 64 sequences of zeros
    fq.prompt_attention(*parts, 1, 1, ends, out=out)
    for lo in (0, at):
        h = host(view[lo:lo + n])
        want, off = ref.grouped(h[:, :D], h[:, D:2 * D], h[:, 2 * D:], 1, 1, 0, D ** -0.5)
        assert_within(host(out[lo:lo + n]), want, off)
    positions, freq = torch.arange(66000, dtype=torch.int32, device=DEV), to_dev((0.9 ** np.arange(64)).astype(np.float32))
    fq.rotate_heads(big, 1, 1, D, positions, freq, out=big)
    after = host(tail[:, :2 * D])
    want, off = ref.rotate(h, 1, 1, D, np.arange(at, at + n), (0.9 ** np.arange(64)).astype(np.float32))
    assert_within(after, want, off)
    del starts, packed


# ---- all of it together ----------------------------------------------------------------------------------------

def test_a_block_with_its_attention():
    """Prompts through a block's stage 0, rotation, attention over the prompt, the cache, and stages 1 to 3; then tokens one at
    a time over the cache.  Each attention is checked on the rows that the block made."""
    rng = np.random.default_rng(18)
    H, F, heads, kv, D = 512, 1024, 4, 2, 128
    QKV = (heads + 2 * kv) * D

    def packed(N, K):
        codes, scales = fq.quant_w6(to_dev((rng.standard_normal((N, K)) / np.sqrt(K)).astype(np.float32)))
        return fq.pack_w6(codes, scales)

    layer = fq.Layer(H, F, QKV, 0, packed(QKV, H), packed(H, H), packed(2 * F, H), packed(H, F),
                     *(to_dev((1 + 0.1 * rng.standard_normal(H)).astype(np.float16)) for _ in range(2)))
    gq, gk = (to_dev((1 + 0.2 * rng.standard_normal(D)).astype(np.float16)) for _ in range(2))
    freq = to_dev((10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32))
    s = Story(rng, 3, kv, D, 32, 140)

    def block(x, parts, prompt):
        M = sum(parts)
        buf = {n: torch.empty((M, w), dtype=torch.float16, device=DEV) for n, w in
               dict(qkv=QKV, attn=H, o=H, x_ffn=H, gate_up=2 * F, down=H).items()}
        ws = layer.make_workspace(M)
        fq.layer_linears(layer, M, ws, 0, 0, x=x, qkv=buf["qkv"])
        positions = np.concatenate([np.arange(len(s.k[i]), len(s.k[i]) + n) for i, n in enumerate(parts)]).astype(np.int32)
        plain = host(buf["qkv"])
        qkv = fq.rotate_heads(buf["qkv"], heads, kv, D, to_dev(positions), freq, gq, gk, out=buf["qkv"])
        want, off = ref.rotate(plain, heads, kv, D, positions, host(freq), host(gq), host(gk))
        rows = host(qkv)
        assert_within(rows[:, :(heads + kv) * D], want, off)
        q, k, v = qkv[:, :heads * D], qkv[:, heads * D:(heads + kv) * D], qkv[:, (heads + kv) * D:]
        at = 0
        for i, n in enumerate(parts):
            s.k[i] = np.concatenate([s.k[i], host(k[at:at + n])])
            s.v[i] = np.concatenate([s.v[i], host(v[at:at + n])])
            at += n
        seqs = s.seqs(parts)
        fq.cache_append(s.cache, k, v, seqs)
        if prompt:
            fq.prompt_attention(q, k, v, heads, kv, seqs.starts, out=buf["attn"])
            check_prompt(host(q), host(k), host(v), parts, heads, kv, host(buf["attn"]), D ** -0.5)
        else:
            fq.cache_attention(s.cache, q, heads, seqs, out=buf["attn"])
            at = 0
            for i, n in enumerate(parts):
                want, off = ref.grouped(host(q)[at:at + n], ref.stored(s.k[i], kv), ref.stored(s.v[i], kv), heads, kv,
                                        len(s.k[i]) - n, D ** -0.5)
                assert_within(host(buf["attn"])[at:at + n], want, off)
                at += n
        fq.layer_linears(layer, M, ws, 1, 1, attn=buf["attn"], o=buf["o"])
        buf["x_ffn"].copy_(x + buf["o"])
        fq.layer_linears(layer, M, ws, 2, 3, x_ffn=buf["x_ffn"], gate_up=buf["gate_up"], down=buf["down"])
        assert torch.isfinite(buf["down"]).all()
        return buf["x_ffn"] + buf["down"]

    x = block(to_dev(normal(rng, 118, H)), [50, 1, 67], True)
    s.check_read([50, 1, 67])
    last = x[[49, 50, 117]].contiguous()
    for step in range(18):
        last = block(last, [1, 1, 1], False)
        last = (last / last.float().square().mean(1, keepdim=True).sqrt()).half()
    last = torch.cat([last, last])
    block(last, [3, 0, 3], False)
    s.check_read([71, 19, 88])
