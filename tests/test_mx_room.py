"""The workspace sizes that the MX binding remembers: the library's own answers, and not more of them the longer a program runs."""
import random
import tracemalloc

import pytest

from paper_2501_17116_amd import binding as b

OPS = [b.FP4_OP_MX_FWD, b.FP4_OP_MX_DGRAD, b.FP4_OP_MX_WGRAD, b.FP4_OP_MX_BWD]


class Room:
    def get(self, nbytes):
        self.asked = nbytes
        return self

    def data_ptr(self):
        return 0

    def numel(self):
        return self.asked


@pytest.fixture
def asked(monkeypatch):
    monkeypatch.setattr(b, "_stream_of", lambda t: 0)
    room = Room()
    return lambda op, M, K, N: b._mx_ws(op, M, K, N, room, None)[1]


def test_answers_are_the_librarys(asked):
    rng = random.Random(1)
    for _ in range(2000):
        q = rng.choice(OPS), rng.randint(0, 5000), rng.randint(0, 5000), rng.randint(0, 5000)
        for _ in range(2):
            assert asked(*q) == b.workspace_bytes(*q, b.FP4_BF16)


def test_a_server_of_many_token_counts_keeps_no_more_of_them(asked):
    for M in range(20000):        # every size there is room for
        asked(b.FP4_OP_MX_FWD, M, 4096, 4096)
    tracemalloc.start()
    try:
        before = tracemalloc.get_traced_memory()[0]
        for M in range(20000, 60000):
            asked(b.FP4_OP_MX_FWD, M, 4096, 4096)
        grown = tracemalloc.get_traced_memory()[0] - before
    finally:
        tracemalloc.stop()
    assert grown < 1 << 20        # an entry takes over a hundred bytes: forty thousand would be four million
