"""A CTA of the chunk attention (csrc/chunk_attn.cu) as six actors -- two softmax groups, two MMA issuers, the K and the V
producer -- over mbarriers with parity semantics, stepped in random order.

It restates the waits and signals of the kernel in the kernel's order, so a change there has to be made here too.  A walk is
a list of pieces (key tiles, two row tiles?) as one CTA meets them.  The outcome names what went wrong:

  stuck     nothing can move and not every actor is done
  early     a wait passed although what it waits for has not happened (a parity taken for the one two before it)
  lapped    a wait passed two completions late: it could as well have been missed
  in flight copies or matrix products under way when the CTA's memory goes back

With `give_up` any wait may run out: the CTA's abort flag goes up, the others leave at their next unready wait, and what is in
flight has to be waited for.  The switches turn back single decisions of the kernel, to show what each of them is for.
"""
from __future__ import annotations

import random


class Bar:
    __slots__ = ("name", "need", "left", "done", "in_flight")

    def __init__(self, name, need):
        self.name, self.need, self.left, self.done, self.in_flight = name, need, need, 0, 0

    def arrive(self):
        self.left -= 1
        assert self.left >= 0, f"more arrivals than counted at {self.name}"
        self.check()

    def check(self):
        if self.left == 0 and self.in_flight == 0:
            self.done += 1
            self.left = self.need

    def passes(self, count):
        """The test of the count-th completion (from 0), by its parity."""
        return (self.done & 1) != (count & 1)


class Cta:
    def __init__(self, pieces, dim, rnd, ragged=0.3, give_up=0.0, counted_when_sent=True, flag_is_final=True, pairs_release_q=True):
        self.pieces, self.rnd, self.ragged, self.give_up = pieces, rnd, ragged, give_up
        self.counted_when_sent, self.flag_is_final, self.pairs_release_q = counted_when_sent, flag_is_final, pairs_release_q
        self.k_stages, self.v_stages = (3, 2) if dim == 128 else (5, 5)
        self.abort = False
        self.copies = []                               # barriers that copies in flight will complete
        self.products = [[], []]                       # per issuer, in order: the barriers each commit arrives at
        self.flushed = [False, False]                  # issuers that waited for their products at the end
        self.bars = {}
        for s in range(self.k_stages):
            self._bar(1, "k_full", s, 0), self._bar(1, "k_full", s, 1), self._bar(2, "k_empty", s)
        for s in range(self.v_stages):
            self._bar(1, "v_full", s, 0), self._bar(1, "v_full", s, 1), self._bar(2, "v_empty", s)
        for s in range(2):
            for name, need in (("land", 1), ("q_full", 1), ("q_empty", 2), ("s_full", 1), ("o_full", 1), ("x_ready", 4), ("x_done", 4), ("begun", 4)):
                self._bar(need, name, s)
            self._bar(4, "p_full", s, 0), self._bar(4, "p_full", s, 1)

    def _bar(self, need, *name):
        self.bars[name] = Bar(name, need)

    def arrive(self, *name, times=1):
        for _ in range(times):
            self.bars[name].arrive()

    def passes(self, name, count):
        return self.bars[name].passes(count)

    def send(self, *name):
        """expect_tx and the copy behind it."""
        b = self.bars[name]
        b.in_flight = 1
        b.arrive()
        self.copies.append(b)

    def land(self, b):
        self.copies.remove(b)
        b.in_flight = 0
        b.check()

    def drain(self, name, count):
        """A bounded wait at the end: it passes at once, or when the barrier's copy lands, or it runs out."""
        b = self.bars[name]
        if not b.passes(count) and b in self.copies:
            self.land(b)

    @staticmethod
    def full(name, tile, stages):
        return (name, tile % stages, (tile // stages) & 1), tile // stages // 2

    # Actors yield (barrier, count) to wait and None to let others go first; a wait answers whether it passed.
    def softmax(self, s):
        n_s = n_o = n_o_other = n_x = n_x_other = tiles = 0
        lent = False
        for n, dual in self.pieces:
            leads, join = dual or (tiles & 1) == s, not dual and n > 1
            first = 0 if leads else 1
            tiles += n & 1
            if not leads and not join:
                n_o_other += n > 0
                continue
            if n > 0 and lent:
                if not (yield ("x_done", s ^ 1), n_x_other):
                    return
                n_x_other, lent = n_x_other + 1, False
            for _ in range(first, n, 1 if dual else 2):
                if not (yield ("s_full", s), n_s):
                    return
                n_s += 1
                if dual:
                    self.arrive("begun", s, times=4)
                yield None
                self.arrive("p_full", s, 0, times=4)
                yield None
                self.arrive("p_full", s, 1, times=4)
            if not leads:
                self.arrive("x_ready", s ^ 1, times=4)
                lent, n_o, n_o_other = True, n_o + 1, n_o_other + 1
                continue
            if n > 0:
                if not (yield ("o_full", s), n_o):
                    return
                n_o += 1
            if join:
                if not (yield ("x_ready", s), n_x) or not (yield ("o_full", s ^ 1), n_o_other):
                    return
                n_x += 1
            n_o_other += join or (dual and n > 0)
            yield None
            if join:
                self.arrive("x_done", s, times=4)

    def issuer(self, s):
        yield from self._issue(s)
        yield "done"
        if self.abort:
            self.flushed[s] = True

    def _issue(self, s):
        n_k = n_p = q_slot = n_begun = 0
        for n, dual in self.pieces:
            if n == 0:
                continue
            mine = (q_slot + (s if dual else 0)) & 1
            if not (yield ("q_full", q_slot & 1), q_slot >> 1):
                return
            if dual and not (yield ("q_full", (q_slot + 1) & 1), (q_slot + 1) >> 1):
                return
            q_slot += 2 if dual else 1
            if dual and self.pairs_release_q:
                self.arrive("q_empty", mine ^ 1)
            step, first = (1, 0) if dual else (2, (n_k ^ s) & 1)
            if first >= n:
                self.arrive("q_empty", mine)
            for i in range(first, n, step):
                tile, last = n_k + i, i + step >= n
                if not (yield self.full("k_full", tile, self.k_stages)):
                    return
                if dual:
                    if s == 1 and not (yield ("begun", 0), n_begun):
                        return
                    if s == 0 and n_begun and not (yield ("begun", 1), n_begun - 1):
                        return
                    n_begun += 1
                commit = [("s_full", s), ("k_empty", tile % self.k_stages)]
                if not dual:
                    self.arrive("k_empty", tile % self.k_stages)
                if last:
                    commit.append(("q_empty", mine))
                    if dual and not self.pairs_release_q:
                        self.arrive("q_empty", mine)
                self.products[s].append(commit)
                if not (yield self.full("v_full", tile, self.v_stages)):
                    return
                for half in range(2):
                    if not (yield ("p_full", s, half), n_p):
                        return
                    if half:
                        if not dual:
                            self.arrive("v_empty", tile % self.v_stages)
                        self.products[s].append([("v_empty", tile % self.v_stages)] + ([("o_full", s)] if last else []))
                n_p += 1
            n_k += n

    def producer(self, is_v):
        name, stages = ("v", self.v_stages) if is_v else ("k", self.k_stages)
        sent = {"tiles": 0, "q": 0, "landings": 0, "by_landing": []}
        yield from self._produce(is_v, name, stages, sent)
        yield "done"
        if not self.abort:
            return
        for back in range(min(stages, sent["tiles"])):
            if not (back < len(sent["by_landing"]) and sent["by_landing"][-1 - back]):
                self.drain(*self.full(name + "_full", sent["tiles"] - 1 - back, stages))
        for back in range(1, 3):
            if back <= sent["landings"]:
                self.drain(("land", (sent["landings"] - back) & 1), (sent["landings"] - back) >> 1)
            if back <= sent["q"]:
                self.drain(("q_full", (sent["q"] - back) & 1), (sent["q"] - back) >> 1)

    def _produce(self, is_v, name, stages, sent):
        n_t, due = 0, None                             # due: landing, full barrier

        def clear():
            nonlocal due
            at, due = due, None
            if not (yield ("land", at[0] & 1), at[0] >> 1):
                return False
            self.arrive(*at[1])
            return True

        def send_q(dual, must):
            last = sent["q"] + (1 if dual else 0)
            for k in range(sent["q"], last + 1):
                if k >= 2:
                    bar, count = ("q_empty", k & 1), (k >> 1) - 1
                    if not ((yield bar, count) if must else self.passes(bar, count)):
                        return False
            for k in range(sent["q"], last + 1):
                self.send("q_full", k & 1)
            sent["q"] = last + 1
            return True

        for n, dual in self.pieces:
            if n == 0:
                continue
            q_sent = is_v or (yield from send_q(dual, False))
            gaps = is_v and self.rnd.random() < self.ragged / 4
            for i in range(n):
                stage, use = n_t % stages, n_t // stages
                if use > 0:
                    if due and not self.passes((name + "_empty", stage), use - 1) and not (yield from clear()):
                        return
                    if not (yield (name + "_empty", stage), use - 1):
                        return
                full = self.full(name + "_full", n_t, stages)[0]
                ragged = gaps or (is_v and self.rnd.random() < self.ragged)
                self.send(*(("land", sent["landings"] & 1) if ragged else full))
                n_t += 1
                sent["by_landing"].append(ragged)
                if self.counted_when_sent:
                    sent["tiles"] = n_t
                yield None
                late = due
                if late and not (yield from clear()):
                    if ragged:
                        sent["landings"] += 1
                    return
                if ragged:
                    due = (sent["landings"], full)
                    sent["landings"] += 1
                if gaps and not (yield from clear()):
                    return
                if not q_sent and i == min(1, n - 1):
                    q_sent = yield from send_q(dual, True)
                    if not q_sent:
                        return
                sent["tiles"] = n_t
        if due:
            yield from clear()

    def run(self):
        rnd = self.rnd
        actors = {"s0": self.softmax(0), "s1": self.softmax(1), "i0": self.issuer(0), "i1": self.issuer(1),
                  "k": self.producer(False), "v": self.producer(True)}
        waits, weight = dict.fromkeys(actors), {k: rnd.choice((1, 1, 4, 20)) for k in [*actors, "copy", "p0", "p1"]}
        ended = set()                                  # actors at the end of their loops
        while actors:
            able = []
            for k in actors:
                w = waits[k]
                if w == "done":
                    if not self.flag_is_final or len(ended) == 6:
                        able.append(k)
                elif w is None or self.passes(*w) or self.abort or (self.give_up and rnd.random() < self.give_up):
                    able.append(k)
            able += ["copy"] * bool(self.copies) + [f"p{s}" for s in range(2) if self.products[s]]
            if not able:
                if self.give_up:
                    continue                           # somebody's wait will run out
                return "stuck"
            k = rnd.choices(able, [weight[a] for a in able])[0]
            if k == "copy":
                self.land(rnd.choice(self.copies))
                continue
            if k in ("p0", "p1"):
                for name in self.products[int(k[1])].pop(0):
                    self.arrive(*name)
                continue
            w, answer = waits[k], None
            if w is not None and w != "done":
                b = self.bars[w[0]]
                answer = b.passes(w[1])
                if answer and b.done <= w[1]:
                    return "early"
                if answer and b.done > w[1] + 1:
                    return "lapped"
                if not answer:
                    self.abort = True                  # ran out, or left since another did
            try:
                waits[k] = actors[k].send(answer)
                if waits[k] == "done":
                    ended.add(k)
            except StopIteration:
                ended.add(k)
                del actors[k]
        if self.abort:
            # products of an issuer that waited for them are complete
            left = any(self.products[s] and not self.flushed[s] for s in range(2)) or self.copies
            return "in flight" if left else "gave up"
        # nobody gave up: what is still under way has been waited for by somebody, or it is a commit that nobody needs
        return "in flight" if self.copies else "ok"


def random_walk(rnd, longest=12):
    return [(rnd.choice((0, 1, 1, 2, 3, 4, 5, rnd.randrange(1, longest))), rnd.random() < 0.4) for _ in range(rnd.randrange(1, longest))]


def walks(seed, count, **switches):
    """Outcomes of `count` random walks and how often each came."""
    rnd, out = random.Random(seed), {}
    for _ in range(count):
        result = Cta(random_walk(rnd), rnd.choice((64, 128)), rnd, rnd.choice((0, 0.3, 1)), **switches).run()
        out[result] = out.get(result, 0) + 1
    return out
