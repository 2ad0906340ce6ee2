"""How far back a sequence of the 8-bit cache may be shortened, and a model of the ring that holds its recent tokens."""
BLOCK, RING = 16, 32


class Lengths:
    """The lengths that a sequence may be shortened to, from what it has been through: any from `least()` on, and multiples of
    a block."""

    def __init__(self):
        self.begin = self.most = self.length = 0     # most: the furthest length, counted since it began anew at `begin`

    def grow(self, n):
        self.length += n
        self.most = max(self.most, self.length)

    def least(self):
        return max(self.begin, BLOCK * (self.most // BLOCK - 1))

    def allowed(self):
        return [n for n in range(self.length + 1) if n >= self.least() or n % BLOCK == 0]

    def cut(self, n):
        assert n in self.allowed()
        if n < self.least():
            self.begin = self.most = n
        self.length = n


class Ring:
    """What an append reads from the ring and writes into it: each token by its position and the append that brought it."""

    def __init__(self):
        self.at, self.tokens, self.appends = [None] * RING, [], 0

    def holds(self, first, last):
        return all(self.at[t % RING] == self.tokens[t] for t in range(first, last))

    def tail(self, length):
        """Whether the unfinished block's tokens of a sequence of this length are there."""
        return self.holds(length // BLOCK * BLOCK, length)

    def append(self, n):
        first, self.appends = len(self.tokens), self.appends + 1
        assert first % BLOCK == 0 or first // BLOCK == (first + n) // BLOCK or self.tail(first)
        self.tokens += [(first + i, self.appends) for i in range(n)]
        for t in range(max(first, BLOCK * (len(self.tokens) // BLOCK - 1)), len(self.tokens)):
            self.at[t % RING] = self.tokens[t]
