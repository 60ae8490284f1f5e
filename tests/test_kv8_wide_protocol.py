"""The wide form of the attention over the 8-bit cache keeps scores where S lay until a tile's weights are stored: no later
product may write there before (the barrier protocol of kv8_protocol_model.py, with that place watched)."""
import random

from kv8_protocol_model import Cta


class Kept(Cta):
    watched = 2                                        # buffers of S

    def product(self):
        kind, tile = self.products[0][0].tag
        if kind == "s" and tile >= self.watched:
            self.want(all(p is not None and p >= tile - self.watched for p in self.p), "S over scores that wait for their weights")
        super().product()


def outcomes(seed, count, cls=Kept, **kw):
    rnd, got = random.Random(seed), {}
    for _ in range(count):
        pieces = []
        for _ in range(rnd.randint(1, 9)):
            n = rnd.choice([0, 1, 1, 2, 3, 4, 5, 9])
            pieces.append((n, [rnd.random() < 0.3 for _ in range(n)]))
        r = cls(pieces, rnd.choice([2, 4]), rnd, **kw).run()
        got[r] = got.get(r, 0) + 1
    return got


def test_a_buffer_of_s_is_left_alone_until_its_tile_s_weights_are_stored():
    assert outcomes(5, 1500) == {"ok": 1500}


def test_one_buffer_would_not_do():
    class One(Kept):
        watched = 1

    assert outcomes(6, 300, One).get("overrun", 0) > 0
