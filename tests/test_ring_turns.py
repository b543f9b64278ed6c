"""The value ring of attention over pages (pages_attend_kernel), in turns.

A place of the ring is waited for by the parity of its turn alone: a wait for turn t also returns while turn t - 1 is still to come, and never if
turn t + 1 has come as well.  So whoever waits for a turn has to know that the one before is over, and no place may be given back before
everyone who waits for it has seen it.  Where a job's tiles are taken by two streams in turn, and the job has an odd number of them, the streams change places
behind it; a stream that waits for its own tiles alone then does not know the turn before.

Nothing of this shows on a GPU but by copies that land out of order, so that the roles are run here as generators: copies land, and products end,
whenever the schedule likes.  Every wait that returns is looked at."""
import random
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2605_13319_b200" / "csrc" / "serving"


class Wrong(Exception):
    pass


class Barrier:
    """Counts arrivals; `done`: phases that are complete."""

    def __init__(self, count):
        self.count, self.left, self.done = count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.done = self.count, self.done + 1

    def wait(self, turn):
        """For phase `turn` (0 the first), as its parity says it."""
        return self.done & 1 != turn & 1

    def check(self, turn):
        if self.done != turn + 1:
            raise Wrong(f"a wait for turn {turn} returned with {self.done} over")


class Cta:
    """Roles of a CTA over jobs of (tiles, both, whole); a role's generator yields (barrier, turn) to wait for, or None to let others go ahead.
    sees_all: a stream that takes every second tile waits for the other's tiles as well, and gives their places back as its own."""

    def __init__(self, rng, jobs, k_slots, v_slots, sees_all):
        self.rng, self.jobs, self.k_slots, self.v_slots, self.sees_all = rng, jobs, k_slots, v_slots, sees_all
        self.k_full, self.k_empty = ([Barrier(n) for _ in range(k_slots)] for n in (1, 2))
        self.v_full, self.v_empty = ([Barrier(n) for _ in range(v_slots)] for n in (1, 2))
        self.q_full, self.q_empty, self.joint = Barrier(2), Barrier(2), Barrier(2)
        self.s_full, self.p_full, self.o_full = ([Barrier(1) for _ in range(2)] for _ in range(3))
        self.held = {}                             # (ring, slot) -> tile that is there
        self.copies = []                           # [ring, slot, tile, barrier, how long it is put off]
        self.issued = [[], []]                     # a stream's products and commits, which end in order

    # ---- roles
    def fetch(self, ring, slots, full, empty):
        for c in range(sum(n for n, _, _ in self.jobs)):
            at, turn = c % slots, c // slots
            if turn:
                yield empty[at], turn - 1
            self.held.pop((ring, at), None)
            self.copies.append([ring, at, c, full[at], self.rng.choice([0, 0, 3, 30, 300])])
            yield None

    def issuer(self, s):
        first, p_turn = 0, 0

        def products(ring, c):
            self.issued[s].append(("use", ring, c))

        def commit(barrier):
            self.issued[s].append(("arrive", barrier))

        def k_wait(c):
            return self.k_full[c % self.k_slots], c // self.k_slots

        def v_wait(c):
            return self.v_full[c % self.v_slots], c // self.v_slots

        for i, (n, both, _) in enumerate(self.jobs):
            step, j0 = (1, 0) if both else (2, s)
            once = both or self.sees_all           # of a value's place: the other stream says so too

            def release(empty, single):
                commit(empty)
                if not single:
                    commit(empty)

            yield self.q_full, i
            if j0 < n:
                yield k_wait(first + j0)
                products("k", first + j0)
                commit(self.s_full[s])
                release(self.k_empty[(first + j0) % self.k_slots], both)
            if j0 + step >= n:
                commit(self.q_empty)

            def see(c):                            # a tile of the other stream's
                yield v_wait(c)
                self.v_empty[c % self.v_slots].arrive()

            for j in range(j0, n, step):
                more, c = j + step < n, first + j
                if self.sees_all and not both and j > 0:
                    yield from see(c - 1)
                yield v_wait(c)
                if more:
                    yield k_wait(c + step)
                yield self.p_full[s], p_turn
                p_turn += 1
                products("v", c)
                if more:
                    products("k", c + step)
                    commit(self.s_full[s])
                else:
                    commit(self.o_full[s])
                release(self.v_empty[c % self.v_slots], once)
                if more:
                    release(self.k_empty[(c + step) % self.k_slots], both)
                if more and j + 2 * step >= n:
                    commit(self.q_empty)
                if self.sees_all and not both and j + 2 == n:
                    yield from see(c + 1)
            if self.sees_all and not both and j0 >= n:
                yield from see(first)
            first += n

    def rows(self, s):
        first = s_turn = o_turn = joint = 0
        self.q_full.arrive()                       # the first job's queries
        for i, (n, both, whole) in enumerate(self.jobs):
            mine = range(0 if both else s, n, 1 if both else 2)
            for j in mine:
                yield self.s_full[s], s_turn
                s_turn += 1
                c = first + j
                if self.rng.random() < 0.3:        # a tile with a border: its values are looked over
                    yield self.v_full[c % self.v_slots], c // self.v_slots
                self.p_full[s].arrive()
            if i + 1 < len(self.jobs):
                yield self.q_empty, i
                self.q_full.arrive()
            if len(mine):
                yield self.o_full[s], o_turn
                o_turn += 1
            if whole and not both:                 # both streams' sums are the job's
                for _ in range(2):
                    self.joint.arrive()
                    yield self.joint, joint
                    joint += 1
            first += n

    # ---- the schedule
    def run(self):
        roles = [self.fetch("k", self.k_slots, self.k_full, self.k_empty), self.fetch("v", self.v_slots, self.v_full, self.v_empty)]
        roles += [r(s) for s in range(2) for r in (self.issuer, self.rows)]
        waits = [next(r, "over") for r in roles]
        while True:
            can = [("role", i) for i, w in enumerate(waits) if w != "over" and (w is None or w[0].wait(w[1]))]
            can += [("copy", c) for c in self.copies] + [("end", s) for s in range(2) if self.issued[s]]
            if not can:
                if any(w != "over" for w in waits):
                    raise Wrong("waits that never end")
                return
            kind, x = self.rng.choice(can)
            if kind == "role":
                if waits[x] is not None:
                    waits[x][0].check(waits[x][1])
                waits[x] = next(roles[x], "over")
            elif kind == "copy":
                x[4] -= 1
                if x[4] < 0 or len(can) == len(self.copies):
                    self.copies.remove(x)
                    self.held[x[0], x[1]] = x[2]
                    x[3].arrive()
            else:
                what = self.issued[x].pop(0)
                if what[0] == "arrive":
                    what[1].arrive()
                elif self.held.get((what[1], what[2] % (self.k_slots if what[1] == "k" else self.v_slots))) != what[2]:
                    raise Wrong(f"products of {what} over another tile")


def _jobs(rng):
    return [(rng.choice([1, 1, 2, 3, 3, 4, 5, 7]), rng.random() < 0.3, rng.random() < 0.5) for _ in range(rng.randint(2, 7))]


SLOTS = [(2, 2), (4, 4), (4, 6), (8, 8)]           # as the kernel's variants have them


@pytest.mark.parametrize("k_slots,v_slots", SLOTS + [(2, 3)])
def test_every_wait_is_for_the_turn_it_means(k_slots, v_slots):
    for seed in range(400):
        rng = random.Random(seed)
        Cta(rng, _jobs(rng), k_slots, v_slots, True).run()


@pytest.mark.parametrize("k_slots,v_slots", SLOTS[:1] + [(2, 3)])
def test_streams_that_wait_for_their_own_tiles_alone_are_found(k_slots, v_slots):
    found = 0
    for seed in range(400):
        rng = random.Random(seed)
        try:
            Cta(rng, _jobs(rng), k_slots, v_slots, False).run()
        except Wrong:
            found += 1
    assert found > 4


def test_the_kernel_waits_so():
    """The model's two lines are the kernel's."""
    text = re.sub(r"//[^\n]*", "", (CSRC / "attend16_pages.cuh").read_text())
    body = text[re.search(r"__global__[^;{]*\bpages_attend_kernel\(", text).end():]
    body = body[:body.find("registers_more()")]
    see = re.search(r"auto see = \[&\]\(const VPlace& v\) \{([^}]*)\}", body)
    assert see and re.search(r"v_there\(v\)", see.group(1)) and re.search(r"mbar_arrive\(smem_u32\(&c\.v_empty\[v\.slot\]\)\)", see.group(1))
    assert re.search(r"if \(!both && j > 0\) see\(VPlace\(tile_no \+ j - 1\)\);\s*if \(!v_there\(v\)", body)
    assert re.search(r"if \(!both && j \+ 2 == n\) see\(VPlace\(tile_no \+ j \+ 1\)\);\s*\}\s*if \(!both && j0 >= n\) see\(VPlace\(tile_no\)\);\s*tile_no \+= n;", body)
    assert re.search(r"umma_commit\(smem_u32\(&c\.v_empty\[v\.slot\]\)\);", body) and not re.search(r"release\(&c\.v_empty", body)
