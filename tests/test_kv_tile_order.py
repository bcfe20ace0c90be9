"""The order of the roles of the attention's tile kernel, on the CPU: a model of its barriers, with the places and parities that the kernel itself asks for
(csrc/kv_order.h, compiled here), and delays put anywhere.  Every wait has to end, and what is read has to be what was meant."""
import heapq
import os
import random
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_05528_b200", "csrc")
TURNS = 4096
NUMBERS = 8                                  # blocks whose numbers are kept (a constant of the kernel; looked up below)


@pytest.fixture(scope="module")
def rings(tmp_path_factory):
    """{ring: [(place, parity) of every turn]}"""
    at = tmp_path_factory.mktemp("order")
    (at / "order.cc").write_text(f"""#include <cstdio>
#include "kv_order.h"
int main() {{
  const uint32_t places[3] = {{kv::UNIT_PLACES, kv::STAGES, kv::Q_PLACES}};
  for (uint32_t p : places)
    for (uint32_t n = 0; n < {TURNS}; ++n) std::printf("%u %u\\n", kv::ring_place(n, p), kv::ring_parity(n, p));
}}
""")
    subprocess.check_call(["g++", "-std=c++17", "-I", CSRC, str(at / "order.cc"), "-o", str(at / "order")])
    lines = [tuple(map(int, x.split())) for x in subprocess.check_output([str(at / "order")], text=True).splitlines()]
    return {name: lines[i * TURNS:(i + 1) * TURNS] for i, name in enumerate(("units", "stages", "q"))}


class Barrier:
    """Arrivals of a phase, and a wait that knows the parity of a phase alone."""

    def __init__(self, count):
        self.count, self.left, self.phase, self.waiting = count, count, 0, []

    def through(self, parity):
        return self.phase & 1 != parity


class Model:
    """One CTA: units [(blocks, halves)].  Roles are generators that yield a time to pass or (barrier, parity) to wait for."""

    def __init__(self, rings, units, seed, bf16=True, walk=lambda n: 0, slow=None, catch_up=False):
        self.rings, self.units, self.bf16, self.walk, self.catch_up = rings, units, bf16, walk, catch_up
        self.rng = random.Random(seed)
        self.slow = slow or {}
        places = {k: 1 + max(p for p, _ in v) for k, v in rings.items()}
        many = lambda n, count: [Barrier(count) for _ in range(n)]
        self.q = many(places["q"], 1)
        self.q1 = Barrier(1)
        self.s_full, self.s_empty = many(2, 1), many(2, 1)
        self.p_full, self.o_done = many(4, 1), many(4, 1)
        self.k_full, self.k_empty = many(places["stages"], 1), many(places["stages"], 1)
        self.v_full, self.v_empty = many(places["stages"], 1), many(places["stages"], 1)
        self.tops = Barrier(2)
        self.r_full, self.r_empty = many(places["units"], 1), many(places["units"], 7)
        # what lies where, to be compared with what was meant
        self.ring, self.factor, self.numbers, self.q_of = [None] * places["units"], [None] * 2, [None] * NUMBERS, [None] * 2
        self.keys, self.values = [None] * places["stages"], [None] * places["stages"]
        self.scores, self.weights = [None] * 2, [None] * 4

    # ---- the clock
    def arrive(self, b):
        b.left -= 1
        assert b.left >= 0
        if b.left == 0:
            b.left = b.count
            b.phase += 1
            for role in b.waiting:
                self.at(role, self.rng.choice((0, 1, self.rng.randrange(3000))))
            b.waiting = []

    def at(self, role, after):
        heapq.heappush(self.queue, (self.now + after, self.rng.random(), role))

    def run(self):
        """The roles that did not come to their end."""
        self.now, self.queue, live = 0, [], {}
        roles = {"walk": self.walker(), "mma": self.products(), "soft0": self.softmax(0), "soft1": self.softmax(1),
                 **{f"{t}{p}": self.copier(p, t == "v") for t in "kv" for p in (0, 1)}}
        pending = {}
        for name, g in roles.items():
            live[name] = g
            self.at(name, 0)
        while self.queue:
            self.now, _, name = heapq.heappop(self.queue)
            if name in pending:
                b, parity = pending[name]
                if not b.through(parity):
                    b.waiting.append(name)
                    continue
                del pending[name]
            try:
                what = next(live[name])
            except StopIteration:
                del live[name]
                continue
            if isinstance(what, tuple):
                pending[name] = what
                self.at(name, 0)
            else:
                self.at(name, what * self.slow.get(name, 1) * self.rng.choice((0.1, 1, 1, 1, self.rng.random() * 4)))
        return sorted(live)

    # ---- the roles
    def done(self, n):
        self.arrive(self.r_empty[self.rings["units"][n][0]])

    def unit(self, n):
        place, parity = self.rings["units"][n]
        yield self.r_full[place], parity
        got = self.ring[place]
        assert got[0] == n
        return got

    def walker(self):
        for n in range(len(self.units) + 1):
            place, parity = self.rings["units"][n]
            yield self.r_empty[place], parity ^ 1
            yield 30 + self.walk(n)
            self.ring[place] = (n, *self.units[n]) if n < len(self.units) else (n, 0, 0)
            self.arrive(self.r_full[place])

    def softmax(self, half):
        block = turn = 0
        for seg in range(TURNS):
            _, count, halves = yield from self.unit(seg)
            if not count:
                return
            yield 2000
            if self.bf16:
                self.arrive(self.tops)
                yield self.tops, seg & 1
            if half == 0:
                self.factor[seg & 1] = seg
            if half >= halves:
                block += count
                self.done(seg)
                continue
            self.q_of[half] = seg
            self.arrive(self.q1 if half else self.q[self.rings["q"][seg][0]])
            for i in range(count):
                place = turn & 1
                yield self.s_full[half], turn & 1
                assert self.scores[half] == block and self.numbers[block % NUMBERS] == (block, seg)
                yield 300
                self.arrive(self.s_empty[half])
                if i and self.rng.random() < 0.3:
                    yield self.o_done[2 * half + (place ^ 1)], (turn - 1) >> 1 & 1
                    assert self.weights[2 * half + (place ^ 1)] is None
                yield 700
                assert self.numbers[block % NUMBERS] == (block, seg) and self.weights[2 * half + place] is None
                self.weights[2 * half + place] = block
                self.arrive(self.p_full[2 * half + place])
                block += 1
                turn += 1
            yield self.o_done[2 * half + (turn - 1 & 1)], (turn - 1) >> 1 & 1
            assert self.weights[2 * half + (turn - 1 & 1)] is None
            yield 5000
            self.done(seg)

    def copier(self, pair, values):
        full, empty, held = (self.v_full, self.v_empty, self.values) if values else (self.k_full, self.k_empty, self.keys)
        seg, behind, more, ahead, of, waited = 0, 0, True, 0, 0, 0
        n, one = pair - 2, False

        def steps(times):
            nonlocal seg, behind, more, ahead
            for _ in range(times):
                if not more:
                    break
                behind -= 1
                if behind >= 0:
                    continue
                _, count, _ = yield from self.unit(seg)
                more = count > 0
                behind = count - 1
                if more:
                    self.done(seg)
                seg += 1
            ahead = seg - 1
        yield from steps(n + 3)
        while True:
            if one:
                place, parity = self.rings["stages"][n]
                if not values:
                    if self.catch_up:
                        while waited <= of:
                            yield self.q[0], waited & 1
                            waited += 1
                    else:
                        at, q_parity = self.rings["q"][of]
                        yield self.q[at], q_parity
                yield empty[place], parity ^ 1
                if not values:
                    assert self.factor[of & 1] == of
                    self.numbers[n % NUMBERS] = (n, of)
                yield 200
                held[place] = n
                self.arrive(full[place])
            if not more:
                return
            one = True
            of = ahead
            yield 600
            yield from steps(2)
            n += 2

    def products(self):
        n, seg1, turn = 0, 0, [0, 0]
        for seg in range(TURNS):
            _, count, halves = yield from self.unit(seg)
            if not count:
                return
            self.done(seg)
            at, parity = self.rings["q"][seg]
            yield self.q[at], parity
            if halves == 2:
                yield self.q1, seg1 & 1
                seg1 += 1
            assert self.q_of[:halves] == [seg] * halves
            for i in range(-1, count):
                after = n + (i >= 0)
                (st2, parity2), (st, parity) = self.rings["stages"][after], self.rings["stages"][n]
                if i + 1 < count:
                    yield self.k_full[st2], parity2
                for h in range(halves):
                    if i >= 0:
                        yield self.s_empty[h], turn[h] & 1
                    if i + 1 < count:
                        assert self.keys[st2] == after
                        yield 100
                        self.scores[h] = after
                        self.arrive(self.s_full[h])
                        if h + 1 == halves:
                            self.arrive(self.k_empty[st2])
                if i < 0:
                    continue
                yield self.v_full[st], parity
                for h in range(halves):
                    place = 2 * h + (turn[h] & 1)
                    yield self.p_full[place], turn[h] >> 1 & 1
                    assert self.values[st] == n and self.weights[place] == n
                    yield 100
                    self.weights[place] = None
                    self.arrive(self.o_done[place])
                    if h + 1 == halves:
                        self.arrive(self.v_empty[st])
                    turn[h] += 1
                n += 1


def stuck(rings, units, seed, **kw):
    try:
        return Model(rings, units, seed, **kw).run()
    except AssertionError:
        return ["what was read"]


ONES = [(1, 1)] * 24
DELAYS = [(entry, cycles) for entry in range(1, 12) for cycles in (20000, 45000, 200000)]


def test_every_wait_ends_when_a_unit_is_long_in_coming(rings):
    """Units of one block, and a walker that steps over hundreds of sequences before one of them."""
    for halves in (1, 2):
        for entry, cycles in DELAYS:
            for seed in range(4):
                assert not stuck(rings, [(1, halves)] * 24, seed, walk=lambda n: cycles * (n == entry))


def test_every_wait_ends_whatever_is_slow(rings):
    rng = random.Random(5)
    for seed in range(400):
        units = [(rng.choice((1, 1, 1, 2, 3, rng.randint(1, 20))), rng.choice((1, 2))) for _ in range(rng.randint(1, 30))]
        slow = {name: rng.choice((1, 1, 1, 5, 40)) for name in ("walk", "mma", "soft0", "soft1", "k0", "k1", "v0", "v1")}
        gaps = {rng.randrange(30): rng.randrange(100000) for _ in range(3)}
        assert not stuck(rings, units, seed, bf16=bool(seed & 1), slow=slow, walk=lambda n: gaps.get(n, 0)), (seed, units)


def test_the_model_sees_a_phase_that_is_looked_for_too_late(rings):
    """With one place for q, and its phases caught up with when there is a block, some of the delays lock the roles up."""
    one = {**rings, "q": [(0, n & 1) for n in range(TURNS)]}
    assert any(stuck(one, ONES, seed, walk=lambda n: cycles * (n == entry), catch_up=True) for entry, cycles in DELAYS for seed in range(4))
    # looking only for the unit in hand is no help there: its parity is that of the unit two before it too
    assert any(stuck(one, ONES, seed, walk=lambda n: cycles * (n == entry)) for entry, cycles in DELAYS for seed in range(4))
    # (two blocks a unit: both pairs take part in each)
    assert not any(stuck(one, [(2, 2)] * 12, seed, walk=lambda n: cycles * (n == entry), catch_up=True) for entry, cycles in DELAYS for seed in range(2))


def test_the_kernel_asks_as_the_model_does():
    text = open(os.path.join(CSRC, "kv_attend_tcgen05.cu")).read()
    code = re.sub(r"//[^\n]*", "", text)
    assert re.search(r"q_bar = \[&\]\(uint32_t n\) \{ return q_full \+ 8 \* ring_place\(n, Q_PLACES\); \}", code)
    # every wait for q, and every arrival, by the unit
    waits = re.findall(r"wait(?:_warp)?\((q\w*[^;]*);", code)
    assert sorted(w.split(",")[0] for w in waits) == ["q1_full", "q_bar(of)", "q_bar(seg)"]
    assert all("ring_parity(" + re.match(r"q_bar\((\w+)\)", w).group(1) + ", Q_PLACES)" in w for w in waits if w.startswith("q_bar"))
    assert re.findall(r"arrive\([^;]*q[^;]*\);", code) == ["arrive(half ? q1_full : q_bar(seg));"]
    assert int(re.search(r"constexpr int NUMBERS = (\d+)", code).group(1)) == NUMBERS
    # barriers by name lie one behind the other
    at = {"q_full": 0}
    for name, base, off in re.findall(r"(\w+_full|\w+_empty|o_done) = (bar0|q_full|r_full)(?: \+ (8 \* Q_PLACES|8 \* RING|\d+))?[,;]", code):
        at[name] = (0 if base == "bar0" else at[base]) + {"": 0, "8 * Q_PLACES": 16, "8 * RING": 32}.get(off, int(off) if off.isdigit() else 0)
    sizes = {"q_full": 2, "q1_full": 1, "s_full": 2, "s_empty": 2, "p_full": 4, "o_done": 4, "k_full": 4, "k_empty": 4, "v_full": 4, "v_empty": 4,
             "t_full": 1, "r_full": 4, "r_empty": 4}
    assert sorted(at) == sorted(sizes)
    end = 0
    for name in sorted(sizes, key=at.get):
        assert at[name] == end, name
        end += 8 * sizes[name]
    assert end == 8 * (32 + 2 * 4) and "bars[32 + 2 * RING]" in code
