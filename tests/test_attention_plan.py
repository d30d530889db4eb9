"""Launches of the attention's passes over all sizes that are accepted."""
import random

from attention_plan import plans


def _calls():
    few = [(1 << 20, 1 << 20, 1 << 20, 8, 8, 8), (1 << 18, 1 << 18, 1 << 18, 32, 32, 64), ((1 << 30) - 1, (1 << 30) - 1, 1, 1, 1, 8),
           ((1 << 30) - 1, (1 << 30) - 1, 1 << 20, 1, 1, 8), (1 << 20, 1 << 20, 1 << 20, 1023, 1, 8), (1 << 20, 5, 1 << 20, 1 << 14, 1 << 14, 8),
           (3, 3, 1 << 20, 1 << 14, 1 << 14, 128), ((1 << 16) - 1, (1 << 30) - 1, 1, 1 << 14, 1, 128), ((1 << 30) - 1, 1 << 10, 3, 1 << 14, 1 << 14, 16), (0, 0, 1, 1, 1, 8)]
    rng = random.Random(5)
    for _ in range(2000):
        kv, group = 1 << rng.randrange(15), 0
        group = 1 << rng.randrange(15 - kv.bit_length() + 1)
        tq, tk = (int(2 ** rng.uniform(0, 30)) for _ in range(2))
        few.append((min(tq, ((1 << 30) - 1) // group), tk, int(2 ** rng.uniform(0, 20)), kv * group, kv, rng.choice((8, 64, 96, 128))))
    return [c + (causal,) for c in few for causal in (0, 1)]


def test_every_size_has_launches(tmp_path):
    """No launch reaches 2^32 threads, together they take all kv heads, and what joins shares is one launch."""
    calls = _calls()
    several = 0
    for call, both in zip(calls, plans(str(tmp_path), calls)):
        for p in both:
            assert p["fits"] == 1, call
            assert p["waves"] in (4, 8) and 1 <= p["shares"] <= 64 and 1 <= p["heads"] <= call[4], (call, p)
            assert p["places"] * p["shares"] * p["heads"] * p["waves"] * 64 < 1 << 32, (call, p)
            assert p["heads"] == call[4] or p["heads"] < 8 or p["heads"] % 8 == 0, (call, p)
            assert p["shares"] == 1 or p["joins"] < 1 << 23, (call, p)
            several += p["heads"] < call[4]
    assert several > 0
