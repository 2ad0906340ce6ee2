"""A block's attention at the edges of what its interface allows, against plain forms in 64 bits (attention_reference)."""
import numpy as np
import pytest

import attention_reference as ref
from cache_ring import Lengths
from gpu_helpers import say
from test_gpu_attention import Story

pytestmark = pytest.mark.gpu


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
