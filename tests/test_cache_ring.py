"""The bound of shortening, on a model of the ring: whatever a sequence has been through, the tokens that a permitted length needs
are in the ring."""
import random

from cache_ring import Lengths, Ring


def test_every_permitted_length_has_its_tokens():
    for seed in range(400):
        rng = random.Random(seed)
        ring, lengths = Ring(), Lengths()
        for _ in range(40):
            n = rng.choice([1, 1, 2, 5, 9, 15, 16, 17, 31, 33, 100])
            ring.append(n)
            lengths.grow(n)
            for length in lengths.allowed():
                assert ring.tail(length), (seed, length)
            if rng.random() < 0.7:
                allowed = lengths.allowed()
                length = rng.choice([allowed[-1], lengths.least(), rng.choice(allowed), rng.choice(allowed[-20:])])
                length = min(length, lengths.length)
                lengths.cut(length)
                del ring.tokens[length:]


def test_cuts_do_not_add_up():
    """100 tokens, cut to 82, 9 more: the bound is that of 100, not that of 91, whose block before lies under tokens 96 to 99."""
    ring, lengths = Ring(), Lengths()
    ring.append(100)
    lengths.grow(100)
    lengths.cut(82)
    del ring.tokens[82:]
    ring.append(9)
    lengths.grow(9)
    assert lengths.least() == 80 and ring.tail(80) and ring.tail(91)
    assert not ring.tail(70) and ring.at[0] == (96, 1)
    lengths.cut(64)                                  # a multiple of a block: the sequence begins anew there
    del ring.tokens[64:]
    ring.append(7)
    lengths.grow(7)
    assert lengths.least() == 64 and all(ring.tail(n) for n in range(64, 72)) and not ring.tail(63)
