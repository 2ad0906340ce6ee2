"""A block's attention at the edges of what its interface allows, against plain forms in 64 bits (attention_reference)."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2508_04405_amd as fq
from cache_ring import Lengths
from gpu_helpers import say, to_dev
from test_gpu_attention import Story, assert_within, host, i32, keys, normal, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("D,page", [(64, 16), (128, 32)])
def test_cuts_one_after_the_other(D, page):
    """Appends and cuts in any order, each cut to a length that the ones before it leave; the lowest one most often."""
    rng = np.random.default_rng([30, D])
    s, lengths, heads = Story(rng, 2, 1, D, page, 480), Lengths(), 4
    s.append([100, 5])
    lengths.grow(100)
    for cut, n in [(82, 9), (80, 1), (64, 7), (64, 40)] + [(None, int(n)) for n in rng.integers(1, 34, 40)]:
        if cut is None:
            allowed = lengths.allowed()
            cut = int(rng.choice([min(lengths.least(), lengths.length), allowed[-1], rng.choice(allowed), rng.choice(allowed[-12:])]))
        say(f"{lengths.length} -> {cut} -> {cut + n}")
        lengths.cut(cut)
        s.cut(0, cut)
        s.check_read([cut, 5])
        if cut:
            s.check_attention([1, 1], heads)
        n = min(n, 480 - cut)
        s.append([n, 0])
        lengths.grow(n)
        s.check_read(s.lengths())
        s.check_attention([min(n, 3), 1], heads)


@pytest.mark.parametrize("kv,D,page", [(1, 64, 16), (2, 128, 32), (3, 64, 64)])
def test_appends_drop_what_the_table_has_no_room_for(kv, D, page):
    rng = np.random.default_rng([31, D, page])
    room, width = 64, kv * D
    s = Story(rng, 2, kv, D, page, room)
    s.append([64, 20])

    def both(parts, lengths):
        return fq.Sequences(starts_of(parts), i32(lengths), to_dev(s.table), to_dev(s.slots))

    # a sequence that has no room left stays as it is
    for n, length in ((1, 65), (1, 66), (16, 80), (40, 104), (5, 2**31 - 1), (3, 2**30), (3, 2**30 + 3)):
        say(f"{n} rows up to {length}")
        codes, recent = s.cache.codes.clone(), s.cache.recent.clone()
        rows = to_dev(normal(rng, n, 2 * width))
        fq.cache_append(s.cache, rows[:, :width], rows[:, width:], both([n, 0], [length, 20]))
        assert torch.equal(s.cache.codes, codes) and torch.equal(s.cache.recent, recent)
        got = torch.full((2, n, width), 5.0, dtype=torch.float16, device=DEV)
        fq.cache_read(s.cache, both([n, 0], [length, 20]), out=(got[0], got[1]))
        assert not host(got).any()
    # of rows that reach across the end of the room, the first ones are taken
    for at, n in ((60, 7), (48, 30), (33, 64), (0, 70), (63, 1), (63, 2)):
        say(f"{n} rows behind {at}")
        s.cut(0, 48 if at > 48 else 0)
        if len(s.k[0]) < at:
            s.append([at - len(s.k[0]), 0])
        k, v = keys(rng, n, width), normal(rng, n, width)
        s.k[0], s.v[0] = (np.concatenate([a, b])[:room] for a, b in ((s.k[0], k), (s.v[0], v)))
        fq.cache_append(s.cache, to_dev(k), to_dev(v), both([n, 0], [at + n, 20]))
        s.check_read(s.lengths())
        s.check_attention([2, 1], 2 * kv)
        s.cut(0, 63)
        s.check_read([63, 20])                       # (from the ring)
        s.append([1, 0])
        got = fq.cache_read(s.cache, both([room + 3, 20], [room + 3, 20]), rows=room + 23)
        for x, rows in zip(got, (s.k, s.v)):
            assert np.array_equal(host(x)[:room], ref.stored_half(rows[0], kv)) and not host(x)[room:room + 3].any()
            assert np.array_equal(host(x)[room + 3:], ref.stored_half(rows[1], kv))


@pytest.mark.parametrize("M", [1, 2])
@pytest.mark.parametrize("norm", [False, True])
def test_rotation_in_place_into_a_part_of_the_row(M, norm):
    """x the fused row, out the part of it that is rotated."""
    rng = np.random.default_rng([32, M])
    heads, kv, D = 4, 2, 64
    width = (heads + kv) * D
    x, positions = normal(rng, M, width + kv * D), np.arange(7, 7 + M, dtype=np.int32)
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    g = normal(rng, D) if norm else None
    want, off = ref.rotate(x, heads, kv, D, positions, freq, g, g)
    gamma = to_dev(g) if norm else None
    dx = to_dev(x)
    fq.rotate_heads(dx, heads, kv, D, to_dev(positions), to_dev(freq), gamma, gamma, out=dx[:, :width])
    assert_within(host(dx)[:, :width], want, off)
    assert np.array_equal(host(dx)[:, width:], x[:, width:])


@pytest.mark.parametrize("eps", [1.4e-45, 1e-39, 1.2e-38])
def test_norm_of_zeros_with_the_smallest_eps(eps):
    rng = np.random.default_rng(33)
    heads, kv, D, M = 3, 1, 64, 5
    x = normal(rng, M, (heads + kv) * D)
    x[1] = 0
    x[3, D:2 * D] = 0
    x[4] *= np.float16(6e-8)
    g, positions = normal(rng, D), np.arange(M, dtype=np.int32)
    freq = (0.9 ** np.arange(D // 2)).astype(np.float32)
    want, off = ref.rotate(x, heads, kv, D, positions, freq, g, g, eps)
    got = host(fq.rotate_heads(to_dev(x), heads, kv, D, to_dev(positions), to_dev(freq), to_dev(g), to_dev(g), eps=eps))
    assert_within(got, want, off)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 3, 10])
@pytest.mark.parametrize("stages", [0, 3])
def test_an_unfinished_block_of_tiny_values(D, new, stages):
    """Equal values of 1e-4, full blocks and an unfinished one whose first key every row prefers by so much that the weights of the
    others, times their scale of 13 * 2^-24, are numbers of few bits.  The mean of equal values is that value."""
    heads, stage = 8, 128 if D == 64 else 64
    length, value = stage * stages + stage - 1, 1651 * 2.0**-24          # 127 codes of that scale
    rng = np.random.default_rng([34, D, new])
    s = Story(rng, 1, 1, D, 16, length + 1)
    for weight in (0.4, 12.45, 12.55, 100.45, 3000.5):                   # of the others: in steps of 2^-33 / 2^-24
        say(f"D={D} new={new} stages={stages} weight={weight}")
        k = np.zeros((length, D), np.float16)
        k[length // 16 * 16, 0] = 1.0
        s.cut(0, 0)
        s.append([length], lambda M, w: (k, np.full((M, w), value, np.float16)))
        q = np.zeros((new, heads * D), np.float16)
        q[:, ::D] = 16.0
        scale = float(np.log(13 * 512 / weight) / 16.0)
        out = host(fq.cache_attention(s.cache, to_dev(q), heads, s.seqs([new]), scale=scale))
        want, off = ref.grouped(q, ref.stored(k, 1), ref.stored(s.v[0], 1), heads, 1, length - new, scale)
        assert np.abs(want - value).max() < 1e-12
        assert_within(out, want, off, f"weight {weight}")
