"""A CTA of the attention over the 8-bit cache (csrc/kv8_attn.cu) as actors -- softmax warps, the MMA issuer, the K and the V
producer, the Q warp -- over mbarriers with parity semantics and the named barrier of the softmax warps, stepped in random order.

It restates the kernel's waits, signals and memory in the kernel's order, so a change there has to be made here too.  A walk is a
list of pieces: key tiles, and whether each tile hides keys (then the softmax warps also wait for V).  The outcome names
what went wrong:

  stuck      nothing can move and not every actor is done
  early      a wait passed although what it waits for has not happened (a parity taken for the one two before it)
  lapped     a wait passed two completions late: it could as well have been missed
  overrun    something read a buffer that does not hold what it should, or wrote one that is still to be read
  in flight  copies or matrix products under way when the CTA's memory goes back

With `give_up` any wait may run out: the CTA's abort flag goes up, the others leave at their next unready wait, the softmax warps
together at their next barrier, and what is in flight has to be waited for.  The switches turn back single decisions of the
kernel, to show what each of them is for.
"""
from __future__ import annotations

import random

WARPS = 3                                              # of softmax; the kernel has eight


class Wrong(Exception):
    pass


class Bar:
    __slots__ = ("name", "need", "left", "done", "in_flight")

    def __init__(self, name, need):
        self.name, self.need, self.left, self.done, self.in_flight = name, need, need, 0, 0

    def arrive(self):
        self.left -= 1
        if self.left < 0:
            raise Wrong("more arrivals than counted at %s" % (self.name,))
        self.check()

    def check(self):
        if self.left == 0 and self.in_flight == 0:
            self.done += 1
            self.left = self.need


class Cta:
    def __init__(self, pieces, stages, rnd, give_up=0.0, agree=True, counted_when_sent=True, p_waits=True, q_waits_softmax=True):
        self.pieces, self.stages, self.rnd, self.give_up = pieces, stages, rnd, give_up
        self.agree, self.counted_when_sent, self.p_waits, self.q_waits_softmax = agree, counted_when_sent, p_waits, q_waits_softmax
        self.abort, self.flushed, self.gave_up = False, False, False
        self.copies, self.products = [], []            # in flight: (bar, effect); in order: (effect, bars)
        self.bars = {}
        for s in range(stages):
            for name, need in (("k_full", 1), ("k_empty", WARPS), ("v_full", 1), ("v_empty", 1)):
                self.bars[name, s] = Bar((name, s), need)
        for s in range(2):
            for name, need in (("q_full", 1), ("q_empty", 1 + (WARPS if q_waits_softmax else 0)), ("s_full", 1)):
                self.bars[name, s] = Bar((name, s), need)
        self.bars["p_full",], self.bars["o_done",] = Bar("p_full", WARPS), Bar("o_done", 1)
        self.k, self.v, self.s, self.q = [None] * stages, [None] * stages, [None, None], [None, None]
        self.p, self.o = [None] * WARPS, None          # tile whose weights each warp has stored; last tile in O
        self.scored = [-1] * WARPS                     # last tile whose scores a warp has read
        self.meeting, self.meet_no, self.flags = set(), 0, [False, False]

    # -- memory
    def want(self, ok, what):
        if not ok:
            raise Wrong("overrun: " + what)

    def passes(self, name, count):
        b = self.bars[name]
        if (b.done & 1) == (count & 1):
            return False
        if b.done <= count:
            raise Wrong("early")
        if b.done > count + 1:
            raise Wrong("lapped")
        return True

    def send(self, name, effect):
        b = self.bars[name]
        b.in_flight += 1
        b.arrive()
        self.copies.append((b, effect))

    def land(self, i):
        b, effect = self.copies.pop(i)
        effect()
        b.in_flight -= 1
        b.check()

    def product(self):
        effect, bars = self.products.pop(0)
        effect()
        for name in bars:
            self.bars[name].arrive()

    # -- actors: yield ("wait", name, count) (the answer: passed or ran out), ("ready", ..) (a look), ("meet",) or None
    def softmax(self, w):
        fail, turn, n_t = [False], [0], 0

        def hold(name, count):
            if not fail[0]:
                fail[0] = not (yield ("wait", name, count))

        def agreed():
            if not self.agree:                         # each by itself
                if fail[0]:
                    return False
                yield ("meet", w)
                return True
            if fail[0]:
                self.flags[turn[0]] = True
            yield ("meet", w)
            fail[0] = self.flags[turn[0]]
            turn[0] ^= 1
            return not fail[0]

        yield from hold(("q_full", 0), 0)
        if not (yield from agreed()):
            return
        for n_q in range(len(self.pieces) + 1):
            self.want(self.q[n_q & 1] == n_q or fail[0], "meta of another piece")
            if n_q == len(self.pieces):
                return
            n, hides = self.pieces[n_q]
            for i in range(n):
                stage, use = n_t % self.stages, n_t // self.stages
                yield from hold(("s_full", n_t & 1), n_t >> 1)
                if not fail[0]:
                    self.want(self.s[n_t & 1] == n_t, "S of another tile")
                    self.want(self.k[stage] == n_t, "scales of another tile")
                self.scored[w] = n_t
                yield None
                self.bars["k_empty", stage].arrive()
                if not (yield from agreed()):
                    return
                if self.rnd.random() < 0.3 and i > 0:  # a reference moves: O is rescaled (every warp does; one stands for all)
                    yield from hold(("o_done",), n_t - 1)
                    if not fail[0]:
                        self.want(self.o == n_t - 1, "O rescaled while a product writes it")
                yield None
                if i > 0 and self.p_waits:
                    yield from hold(("o_done",), n_t - 1)
                if not fail[0]:
                    self.want(not any(kind == "pv" for kind, _ in self._pending()), "P stored while a product reads it")
                self.p[w] = n_t
                if hides[i]:
                    yield from hold(("v_full", stage), use)
                    if not fail[0]:
                        self.want(self.v[stage] == n_t, "rows of another V cleared")
                yield None
                self.bars["p_full",].arrive()
                n_t += 1
            if n:
                yield ("meet", w)                      # the rows' sums
                yield from hold(("o_done",), n_t - 1)
            yield from hold(("q_full", (n_q + 1) & 1), (n_q + 1) >> 1)
            if not (yield from agreed()):
                return
            if n:
                self.want(self.o == n_t - 1, "rows written before their last tile")
                yield None
                self.want(self.o == n_t - 1 and self.q[n_q & 1] == n_q, "rows overwritten before they are out")
            if self.q_waits_softmax:
                self.bars["q_empty", n_q & 1].arrive()

    def _pending(self):
        return [e.tag for e, _ in self.products]

    def issuer(self):
        n_s = n_p = n_q = 0
        i = n = 0
        owner = {}

        def begin():
            nonlocal n_q, i, n
            while True:
                if not (yield ("wait", ("q_full", n_q & 1), n_q >> 1)):
                    return False
                self.want(self.q[n_q & 1] == n_q, "meta of another piece")
                n = self.pieces[n_q][0] if n_q < len(self.pieces) else -1
                n_q += 1
                i = 0
                if n:
                    return True
                self.bars["q_empty", (n_q - 1) & 1].arrive()

        def issue_s():
            nonlocal n_s, i
            stage, slot, tile, piece = n_s % self.stages, (n_q - 1) & 1, n_s, n_q - 1
            if not (yield ("wait", ("k_full", stage), n_s // self.stages)):
                return False

            def effect():
                self.want(self.k[stage] == tile, "S of another K")
                self.want(self.q[slot] == piece, "S of another Q")
                self.want(tile < 2 or all(x >= tile - 2 for x in self.scored), "S over scores not read yet")
                self.s[tile & 1] = tile
            effect.tag = ("s", tile)
            self.products.append((effect, [("s_full", tile & 1)] + ([("q_empty", slot)] if i + 1 == n else [])))
            owner[tile] = piece
            n_s, i = n_s + 1, i + 1
            return True

        if not (yield from begin()):
            return
        if n < 0 or not (yield from issue_s()):
            return
        while n_p < n_s:
            last, gone = i == n, True
            if not last:
                gone = yield ("ready", ("k_full", n_s % self.stages), n_s // self.stages)
                if gone and not (yield from issue_s()):
                    return
            stage, tile = n_p % self.stages, n_p
            if not (yield ("wait", ("v_full", stage), n_p // self.stages)) or not (yield ("wait", ("p_full",), n_p)):
                return

            def effect(stage=stage, tile=tile):
                self.want(self.v[stage] == tile, "a product with another V")
                self.want(all(x == tile for x in self.p), "a product with other weights")
                self.o = tile
            effect.tag = ("pv", tile)
            self.products.append((effect, [("v_empty", stage), ("o_done",)]))
            n_p += 1
            if not gone:
                if not (yield from issue_s()):
                    return
            elif last and n >= 0:
                if not (yield from begin()):
                    return
                if n < 0:
                    return
                if not (yield from issue_s()):
                    return

    def producer(self, what):
        n_t = 0
        self.sent = getattr(self, "sent", {})
        self.sent[what] = 0
        store = self.k if what == "k" else self.v
        for n, _ in self.pieces:
            for _ in range(n):
                stage, use, tile = n_t % self.stages, n_t // self.stages, n_t
                if use > 0 and not (yield ("wait", (what + "_empty", stage), use - 1)):
                    return

                def effect(stage=stage, tile=tile):
                    store[stage] = tile
                self.want(what == "v" or tile < self.stages or all(x >= tile - self.stages for x in self.scored), "K over scales not read yet")
                self.want(not any(t == (("s" if what == "k" else "pv"), tile - self.stages) for t in self._pending()), "a copy over an operand")
                self.send((what + "_full", stage), effect)
                if self.counted_when_sent:
                    self.sent[what] += 1
                yield None
                if self.rnd.random() < 0.2 and not (yield ("wait", (what + "_full", stage), use)):      # (nothing in the kernel: only delay)
                    return
                if not self.counted_when_sent:
                    self.sent[what] += 1
                n_t += 1

    def q_warp(self):
        for n_q in range(len(self.pieces) + 1):
            if n_q >= 2 and not (yield ("wait", ("q_empty", n_q & 1), (n_q >> 1) - 1)):
                return
            self.want(not any(kind == "s" and self._piece(t) == n_q - 2 for kind, t in self._pending()), "Q over an operand")
            self.q[n_q & 1] = ("being written", n_q)
            yield None
            self.q[n_q & 1] = n_q
            self.bars["q_full", n_q & 1].arrive()

    def _piece(self, tile):
        at = 0
        for k, (n, _) in enumerate(self.pieces):
            at += n
            if tile < at:
                return k
        return len(self.pieces)

    # -- stepping
    def run(self):
        actors = {("softmax", w): self.softmax(w) for w in range(WARPS)}
        actors.update({("issuer",): self.issuer(), ("k",): self.producer("k"), ("v",): self.producer("v"), ("q",): self.q_warp()})
        asked = {a: None for a in actors}
        answer = {a: None for a in actors}
        try:
            self._loop(actors, asked, answer)
        except Wrong as e:
            return str(e).split(":")[0]
        # the end: each producer drains what it counted, the issuer its products
        if self.abort:
            for what in ("k", "v"):
                for back in range(1, min(self.stages, self.sent[what]) + 1):
                    c = self.sent[what] - back
                    b = self.bars[what + "_full", c % self.stages]
                    for i, (bar, _) in enumerate(list(self.copies)):
                        if bar is b:
                            self.copies.pop(next(k for k, (x, _) in enumerate(self.copies) if x is b))
                            break
            self.products = []                         # flushed by a commit of its own
        return "in flight" if self.copies or self.products else ("gave up" if self.abort else "ok")

    def _loop(self, actors, asked, answer):
        while actors or ((self.copies or self.products) and not self.abort):
            moves = []
            if self.copies:
                moves.append("land")
            if self.products:
                moves.append("product")
            for a, want in asked.items():
                if a not in actors:
                    continue
                if want is None or want[0] == "ready":
                    moves.append(a)
                elif want[0] == "wait":
                    if self.passes(want[1], want[2]) or self.abort or (self.give_up and self.rnd.random() < self.give_up):
                        moves.append(a)
            if not moves:
                raise Wrong("stuck")
            m = self.rnd.choice(moves)
            if m == "land":
                self.land(self.rnd.randrange(len(self.copies)))
            elif m == "product":
                try:
                    self.product()
                except Wrong:
                    if not self.abort:                 # after giving up a product may read anything: its results are void
                        raise
            else:
                self._step(m, actors, asked, answer)

    def _step(self, a, actors, asked, answer):
        want = asked[a]
        if want is not None and want[0] == "wait":
            answer[a] = self.passes(want[1], want[2])
            if not answer[a]:
                self.abort = True
        elif want is not None and want[0] == "ready":
            answer[a] = self.passes(want[1], want[2])
        else:
            answer[a] = None
        try:
            asked[a] = actors[a].send(answer[a])
        except StopIteration:
            del actors[a]
            asked[a] = None
            return
        except Wrong:
            if not self.abort:
                raise
            del actors[a]                              # results are void; only getting stuck and what is left in flight count
            asked[a] = None
            return
        if asked[a] is not None and asked[a][0] == "meet":
            self.meeting.add(a)
            if len(self.meeting) == WARPS:
                for b in self.meeting:
                    asked[b] = None
                self.meeting = set()


def walks(seed, count, **kw):
    """Outcomes of `count` random walks of 1 to 9 pieces."""
    rnd, got = random.Random(seed), {}
    for _ in range(count):
        pieces = []
        for _ in range(rnd.randint(1, 9)):
            n = rnd.choice([0, 1, 1, 2, 3, 4, 5, 9])
            pieces.append((n, [rnd.random() < 0.3 for _ in range(n)]))
        r = Cta(pieces, rnd.choice([2, 4]), rnd, **kw).run()
        got[r] = got.get(r, 0) + 1
    return got
