"""The barriers between the warps of attend_rows_kernel, as a model on the CPU: any role delayed at any place, no waiter ever falls two phases behind and
all of them end.

A wait names a phase by its parity. Where a barrier may complete two phases while a role stands in front of its test, the role waits for a phase that is long over, and
mostly everybody else then waits for that role. Such an order works as long as the timing is kind, so it is looked for here and not on a GPU. The roles below are those of the
kernel, a yield for every wait; copies land and commits of products arrive when the schedule says so (commits in their order). ``Order`` has the orders that were
found wrong beside the one that is used, and ``test_the_kernel_waits_and_arrives_in_this_order`` holds the kernel's source to it.
"""
import itertools
import os
import random
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PIECES, MASKS, WARPS = 4, 8, 2                             # (two rows' warps a half stand for four)


class Late(Exception):
    """A role tested for a phase behind which the barrier had already completed another one."""


class Barrier:
    def __init__(self, name, count):
        self.name, self.count, self.left, self.done = name, count, count, 0

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.done, self.left = self.done + 1, self.count

    def passed(self, phase):
        if self.done >= phase + 2:
            raise Late(f"{self.name}: phase {phase} of {self.done}")
        return self.done > phase


class Order:
    """end: the last values of a piece are announced on a barrier of their own ("own") or on that of its logits ("logits").
    keys: the next keys' buffer is tested in every turn of the products ("twice") or in that which takes it ("once")."""

    def __init__(self, end="own", keys="once"):
        self.end, self.keys = end, keys


class Kernel:
    """pieces: (stage, 64s of keys, first tile that is looked through). rescale: whether a rows' warp moves its reference, a function."""

    def __init__(self, pieces, slots, order, rescale):
        self.pieces, self.slots, self.order, self.rescale = pieces, slots, order, rescale
        b = lambda name, count, *shape: self._many(name, count, shape)  # noqa: E731
        self.kv_full, self.kv_empty = b("kv_full", 1, slots), b("kv_empty", 1, slots)
        self.q_full, self.q_empty = b("q_full", 1, 2), b("q_empty", 1, 2)
        self.s_full, self.p_full = b("s_full", 1, 2, 2), b("p_full", WARPS, 2, 2)
        self.o_full, self.o_empty = b("o_full", 1, 2), b("o_empty", WARPS, 2)
        self.piece_full, self.piece_empty = b("piece_full", 1, PIECES), b("piece_empty", 2 * WARPS + 3, PIECES)
        self.mask_full = b("mask_full", 1, MASKS)
        self.scan, self.scanned = Barrier("scan", 1), Barrier("scanned", 1)
        self.landing, self.commits = [], []               # barriers that copies, and products, arrive on later
        self.roles = [("keys", self.keys_()), ("values", self.values_()), ("products", self.products_()), ("scan", self.scan_())]
        self.roles += [(f"rows {h}.{w}", self.rows_(h)) for h in range(2) for w in range(WARPS)]

    def _many(self, name, count, shape):
        if not shape:
            return Barrier(name, count)
        return [self._many(f"{name}[{i}]", count, shape[1:]) for i in range(shape[0])]

    # ---- roles: each yields a list of (barrier, phase) that it tests until all have passed
    def numbered(self):
        """(number, entry of the ring, its round, piece)"""
        for n, x in enumerate(self.pieces + [None]):
            yield n % PIECES, n // PIECES, x

    def keys_(self):
        q_phase, kv = [-1, -1], 0
        for at, turn, x in self.numbered():
            yield [(self.piece_empty[at], turn - 1)]
            self.piece_full[at].arrive()
            if x is None or x[1] == 0:
                continue
            stage, subs, _ = x
            for half in ((0, 1) if stage == 2 else (stage,)):
                yield [(self.q_empty[half], q_phase[half])]
                q_phase[half] += 1
            self.landing.append(self.q_full[0 if stage == 2 else stage])
            if stage == 2:
                self.q_full[1].arrive()
            for _ in range((subs + 1) // 2):
                yield [(self.kv_empty[kv % self.slots], kv // self.slots - 1)]
                self.landing.append(self.kv_full[kv % self.slots])
                yield []                                   # (the mask is told behind the copies)
                self.mask_full[kv // 2 % MASKS].arrive()
                kv += 2

    def values_(self):
        kv = 1
        for at, turn, x in self.numbered():
            yield [(self.piece_full[at], turn)]
            self.piece_empty[at].arrive()
            for _ in range((x[1] + 1) // 2 if x else 0):
                yield [(self.kv_empty[kv % self.slots], kv // self.slots - 1)]
                self.landing.append(self.kv_full[kv % self.slots])
                kv += 2

    def scan_(self):
        n = 0
        for at, turn, x in self.numbered():
            yield [(self.piece_full[at], turn)]
            if x is None:
                return
            for _ in range(max(x[2], 0), (x[1] + 1) // 2):
                yield [(self.scan, n)]
                n += 1
                yield []
                self.scanned.arrive()
            self.piece_empty[at].arrive()

    def products_(self):
        commit = self.commits.append
        kv, q_n, o_n, p_n, scans = 0, [0, 0], [-1, -1], [[0, 0], [0, 0]], 0
        for at, turn, x in self.numbered():
            yield [(self.piece_full[at], turn)]
            self.piece_empty[at].arrive()
            if x is None:
                return
            stage, subs, scan = x
            if subs == 0:
                continue
            halves = (0, 1) if stage == 2 else (stage,)
            for h in halves:
                yield [(self.q_full[h], q_n[h])]
                q_n[h] += 1
            yield [(self.kv_full[kv % self.slots], kv // self.slots)]
            for sub in range(min(2, subs)):
                for h in halves:
                    commit(self.s_full[h][sub])
            commit(self.kv_empty[kv % self.slots])
            if subs <= 2:
                for h in halves:
                    commit(self.q_empty[h])
            kv += 1
            for h in halves:
                yield [(self.o_empty[h], o_n[h])]
                o_n[h] += 1
            for u in range(subs):
                if u % 2 == 0:
                    v = k = kv
                    kv += 1
                    if u + 2 < subs:
                        k = kv
                        kv += 1
                    if u >= 2 * scan:
                        yield [(self.kv_full[v % self.slots], v // self.slots)]
                        self.scan.arrive()
                        yield [(self.scanned, scans)]
                        scans += 1
                waits = [(self.kv_full[v % self.slots], v // self.slots)]
                if self.order.keys == "twice" or u % 2 == 0:
                    waits.append((self.kv_full[k % self.slots], k // self.slots))
                yield waits + [(self.p_full[h][u % 2], p_n[h][u % 2]) for h in halves]
                for h in halves:
                    p_n[h][u % 2] += 1
                for h in halves:
                    commit(self.s_full[h][u % 2] if u + 1 < subs or self.order.end == "logits" else self.o_full[h])
                    if u + 3 == subs:
                        commit(self.q_empty[h])
                if u % 2 == 1 or u + 1 == subs:
                    commit(self.kv_empty[v % self.slots])
                if u + 2 < subs and (u % 2 == 1 or u + 3 == subs):
                    commit(self.kv_empty[k % self.slots])

    def rows_(self, half):
        tile, s_n, o_n = 0, [0, 0], 0
        for at, turn, x in self.numbered():
            yield [(self.piece_full[at], turn)]
            if x is None:
                return
            stage, subs, _ = x
            if stage in (half, 2):
                for u in range(subs):
                    n = tile + u // 2
                    yield [(self.mask_full[n % MASKS], n // MASKS), (self.s_full[half][u % 2], s_n[u % 2])]
                    s_n[u % 2] += 1
                    if u > 0 and self.rescale():
                        yield [(self.s_full[half][u % 2 ^ 1], s_n[u % 2 ^ 1])]
                    self.p_full[half][u % 2].arrive()
                if self.order.end == "logits":
                    for sub in range(min(2, subs)):
                        yield [(self.s_full[half][sub], s_n[sub])]
                        s_n[sub] += 1
                elif subs > 0:
                    yield [(self.o_full[half], o_n)]
                    o_n += 1
                    if subs > 1:
                        s_n[subs % 2] += 1                 # (its last phase was there before; no wait for it unless a reference moved)
                yield []                                   # O is read
                if subs > 0:
                    self.o_empty[half].arrive()
            tile += (subs + 1) // 2
            self.piece_empty[at].arrive()

    # ---- schedules
    def run(self, pick, stalled=None):
        """stalled: (role, n): the role stands in front of its n-th wait until nothing else moves. pick(n): which of n things that can happen does. Returns how
        many waits each role made."""
        counts, waiting, held = {}, {}, stalled
        for name, role in self.roles:
            waiting[name], counts[name] = next(role), 0
        roles = dict(self.roles)
        while True:
            can = []
            for name, wait in waiting.items():
                if held is not None and held == (name, counts[name]):
                    continue
                if all([bar.passed(phase) for bar, phase in wait]):
                    can.append(name)
            if self.commits:
                can.append("commit")
            can += [("landing", i) for i in range(len(self.landing))]
            if not can:
                if held is not None and held[0] in waiting and counts[held[0]] == held[1]:
                    held = None
                    continue
                assert not waiting, f"nothing moves: {[(n, [(b.name, p, b.done) for b, p in w]) for n, w in waiting.items()]}"
                return counts
            what = can[pick(len(can))]
            if what == "commit":
                self.commits.pop(0).arrive()
            elif isinstance(what, tuple):
                self.landing.pop(what[1]).arrive()
            else:
                counts[what] += 1
                try:
                    waiting[what] = next(roles[what])
                except StopIteration:
                    del waiting[what]


def kinds():
    """Pieces: on either half or both, none to six 64s of keys, looked through from the first tile, the second, or not at all."""
    return [(stage, subs, scan) for stage in (0, 1, 2) for subs in (0, 1, 2, 3, 4, 5, 6) for scan in (-1, 1, 9)]


def sequences():
    rng = random.Random(1)
    some = [[(s, n, 9), (t, m, 9), (2, 4, 9)] for (s, t) in ((0, 2), (2, 2), (0, 0), (0, 1), (2, 1)) for n, m in ((1, 2), (3, 3), (4, 5), (5, 1))]
    return some + [[rng.choice(kinds()) for _ in range(rng.randint(1, 7))] for _ in range(12)]


def walk(pieces, slots, order, rescale, delays=None):
    """With nobody delayed, then each role at each of its waits (delays: at so many of them, at random)."""
    rng = random.Random(len(pieces) * 100 + slots)
    make = lambda: Kernel(pieces, slots, order, rescale)  # noqa: E731
    counts = make().run(lambda n: rng.randrange(n))
    places = [(name, i) for name, n in counts.items() for i in range(n)]
    for stalled in places if delays is None else rng.sample(places, min(delays, len(places))):
        make().run(lambda n: 0, stalled)                  # roles first, copies last
        make().run(lambda n: n - 1, stalled)              # copies and commits first
        make().run(lambda n: rng.randrange(n), stalled)


@pytest.mark.parametrize("slots", [5, 10])
@pytest.mark.parametrize("rescale", ["never", "always", "some"])
def test_no_role_falls_two_phases_behind(slots, rescale):
    rng = random.Random(2)
    move = {"never": lambda: False, "always": lambda: True, "some": lambda: rng.random() < 0.3}[rescale]
    for pieces in sequences():
        walk(pieces, slots, Order(), move, 20)


@pytest.mark.parametrize("slots", [5, 10])
def test_every_place_of_every_role(slots):
    for stages, subs in itertools.product(((2, 2, 2), (0, 0, 2), (0, 2, 1)), ((1, 3, 2), (4, 5, 3))):
        walk([(s, n, 1) for s, n in zip(stages, subs)], slots, Order(), lambda: True)


def found(order):
    """Sequences of pieces in which some delay makes a role late, or leaves all of them waiting."""
    late = []
    for pieces in sequences():
        try:
            walk(pieces, 5, order, lambda: False)
        except (Late, AssertionError) as e:
            late.append((pieces, str(e)))
    return late


def test_last_values_announced_where_logits_are_make_rows_late():
    """What the kernel did: the next piece's logits complete the barrier once more in front of a warp that has not yet seen the last one's end."""
    late = found(Order(end="logits"))
    assert late and all("s_full" in why for _, why in late)


def test_keys_tested_behind_their_return_make_the_products_late():
    """What the kernel did with an odd number of 64s of keys: the last turn but two gives the buffer back, the next one tested it again."""
    late = found(Order(keys="twice"))
    assert late and all("kv_full" in why for _, why in late) and all(any(subs % 2 for _, subs, _ in pieces) for pieces, _ in late)


ORDER = {   # every wait (w), arrival (a) and commit (c) in the text, one after the other
    "block": "c s_full c o_full c q_empty c kv_empty c kv_empty",
    "piece": "w q_full w q_full w kv_full c s_full c kv_empty c q_empty w o_empty w o_empty w kv_full a scan w scanned "
             "w kv_full w kv_full w p_full w p_full w kv_full w kv_full w p_full w p_full",
    "softmax_rows": "w s_full a piece_empty w mask_full w s_full w mask_full a p_full w o_full a o_empty a piece_empty",
}


def told(name):
    """The barriers that a function of attend_rows.cu waits for, arrives on and commits to."""
    code = open(os.path.join(ROOT, "paper_2502_00299_b200", "csrc", "attend_rows.cu")).read()
    code = re.sub(r"//[^\n]*", "", code)
    at = re.search(r"(?:bool|void) " + name + r"\(", code).start()
    depth, end = 0, code.index("{", at)
    for end in range(end, len(code)):
        depth += {"{": 1, "}": -1}.get(code[end], 0)
        if depth == 0:
            break
    out = []
    for m in re.finditer(r"(umma_commit|mbar_arrive|mbar_try_wait|wait_warp|\bwait)\(((?:[^()]|\((?:[^()]|\([^()]*\))*\))*)\)", code[at:end]):
        for bar in re.findall(r"sm\.(\w+_full|\w+_empty|scan(?:ned)?)\b", m[2]):
            out.append(({"umma_commit": "c", "mbar_arrive": "a"}.get(m[1], "w")) + " " + bar)
    return " ".join(out)


@pytest.mark.parametrize("name", sorted(ORDER))
def test_the_kernel_waits_and_arrives_in_this_order(name):
    assert told(name) == ORDER[name]


def test_the_kernel_tests_the_next_keys_in_the_turn_that_takes_them():
    code = open(os.path.join(ROOT, "paper_2502_00299_b200", "csrc", "attend_rows.cu")).read()
    tests = re.findall(r"(.{0,20})\b(?:mbar_try_wait\(smem_u32\(&sm\.kv_full\[k_slot\]\)|wait\(sm\.kv_full\[k_slot\])", code)
    assert len(tests) == 2 and all(before.endswith("(u & 1) != 0 || ") for before in tests)
