"""The tree attention kernel's pipeline as a protocol (CPU): its threads, its
ring of tiles and its barriers with their phase parities, run with every copy
held back in turn until nothing else can move.

A wait on an mbarrier names a phase's parity alone, so it also passes while the
phase before that one is still open.  A wait that passes before its own phase
is complete reads a slot that holds something else; the model knows the phase
that every wait means, and counts those that passed too early.
"""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_2606_01563_gb300", "csrc", "tree_step.cu")).read()


class Bar:
    def __init__(self, count=1):
        self.count, self.left, self.phase = count, count, 0  # phase: completed phases

    def arrive(self):
        self.left -= 1
        if self.left == 0:
            self.left, self.phase = self.count, self.phase + 1

    def passes(self, parity):
        return (self.phase & 1) != parity


class Model:
    """segments: (key tiles, slots of C', tiles of which the V rows are touched by the softmax groups)."""

    def __init__(self, slots, blocks, segments, held, known):
        self.NS, self.blocks, self.segs, self.held, self.known = slots, blocks, segments, held, known
        self.full = [Bar() for _ in range(slots)]
        self.empty = [Bar(blocks) for _ in range(slots)]
        two = lambda: [Bar(), Bar()]  # noqa: E731
        self.s_full, self.p_ready, self.turn, self.p_half = two(), two(), two(), two()
        self.q_full, self.q_empty, self.c_grant, self.c_full, self.o_full = Bar(), Bar(4), Bar(), Bar(), Bar(2)
        self.sync = Bar(2)  # the named barrier of the two softmax groups
        self.early = []     # waits that passed before their phase was complete
        self.landing, self.copies = [], 0
        self.turn[0].arrive()

    def geometry(self, seg):
        n, c, touched = seg
        c_tile = max(0, n - (2 if self.blocks == 1 else 1))
        return n, c, touched, c_tile, (lambda j: 2 * j + (c if j >= c_tile else 0)), 2 * c_tile, 2 * n + c

    def copy(self, bar):
        me = self.copies
        self.copies += 1
        if me == self.held:
            self.landing.append(bar)
        else:
            bar.arrive()

    # a wait: (barrier, index of the phase it means, what for)
    def tma(self):
        seq, nq, c_last = 0, 0, -1
        for seg in self.segs:
            n, c, _, c_tile, _, _, _ = self.geometry(seg)
            q_due = True

            def take():
                i = seq % self.NS
                return [(self.empty[i], seq // self.NS - 1, "empty")] if seq >= self.NS else []
            for j in range(n + 1):
                if q_due and (j != 0 or j == n or nq == 0 or self.q_empty.passes((nq - 1) & 1)):
                    if nq > 0:
                        yield self.q_empty, nq - 1, "q_empty"
                    self.copy(self.q_full)
                    nq, q_due = nq + 1, False
                if j == c_tile and c > 0:
                    if c_last >= 0 and seq <= c_last + self.NS:
                        yield self.empty[c_last % self.NS], c_last // self.NS, "last C'"
                    for _ in range(c):
                        yield from take()
                        self.full[seq % self.NS].arrive()
                        seq += 1
                    c_last = seq - 1
                    self.c_grant.arrive()
                if j == n:
                    break
                for _ in range(2):
                    yield from take()
                    self.copy(self.full[seq % self.NS])
                    seq += 1

    def mma(self, g):
        seq = q = c_n = p_n = f_n = 0
        half, reads_c, step = self.blocks == 2, self.blocks == 2 or g == 0, 1 if self.blocks == 2 else 2
        read = False
        for seg in self.segs:
            n, c, _, c_tile, slot, c_slot, total = self.geometry(seg)
            yield self.q_full, q, "Q"
            q += 1
            if read and reads_c:
                if half:
                    yield self.p_ready[g], f_n, "Q C' read"
                    f_n += 1
                else:
                    yield self.p_ready[g], p_n, "Q C' read"
                    p_n += 1
            read = False
            t = 0 if self.blocks == 2 else g
            if t < n:
                at = seq + slot(t)
                yield self.full[at % self.NS], at // self.NS, f"K {t}"
                self.s_full[g].arrive()
                self.empty[at % self.NS].arrive()
            while t < n:
                at = seq + slot(t) + 1
                yield (self.p_half if half else self.p_ready)[g], p_n, "P"
                p_n += 1
                yield self.full[at % self.NS], at // self.NS, f"V {t}"
                if half:
                    yield self.p_ready[g], f_n, "P"
                    f_n += 1
                self.empty[at % self.NS].arrive()
                t += step
                if t < n:
                    at = seq + slot(t)
                    if self.known and self.blocks == 1 and c == 1 and at >= self.NS:
                        yield self.empty[at % self.NS], at // self.NS - 1, f"slot of K {t}"
                    yield self.full[at % self.NS], at // self.NS, f"K {t}"
                    self.s_full[g].arrive()
                    self.empty[at % self.NS].arrive()
            if c > 0:
                if reads_c:
                    yield self.c_full, c_n, "C'"
                    c_n += 1
                    for k in range(c):
                        self.empty[(seq + c_slot + k) % self.NS].arrive()
                read = True
            seq += total
            self.q_empty.arrive()
            self.o_full.arrive()

    def c_warps(self):
        n = 0
        for seg in self.segs:
            if seg[1]:
                yield self.c_grant, n, "C' slots"
                n += 1
                self.c_full.arrive()

    def softmax(self, g):
        nq = ns = no = tn = seq = syncs = 0
        for seg in self.segs:
            n, c, touched, _, slot, _, total = self.geometry(seg)
            if c:
                self.sync.arrive()
                yield self.sync, syncs, "sync"
                syncs += 1
                yield self.q_full, nq, "Q"
            nq += 1
            self.q_empty.arrive()
            for turn in range(n if self.blocks == 2 else (n + 1) >> 1):
                j = turn if self.blocks == 2 else 2 * turn + g
                if j >= n:
                    yield self.turn[g], tn, "turn"
                    tn += 1
                    self.turn[g ^ 1].arrive()
                    break
                yield self.s_full[g], ns, f"S {j}"
                ns += 1
                yield self.turn[g], tn, "turn"
                tn += 1
                if j in touched:
                    at = seq + slot(j) + 1
                    yield self.full[at % self.NS], at // self.NS, f"V {j} touched"
                if self.blocks == 2:
                    self.p_half[g].arrive()
                self.p_ready[g].arrive()
                self.turn[g ^ 1].arrive()
            seq += total
            yield self.o_full, no, "O"
            no += 1
            self.sync.arrive()
            yield self.sync, syncs, "sync"
            syncs += 1
            if c and (self.blocks == 2 or g == 0):
                self.p_ready[g].arrive()

    def run(self):
        threads = [self.tma(), self.mma(0), self.mma(1), self.c_warps(), self.softmax(0), self.softmax(1)]
        waits = [next(t, None) for t in threads]
        while any(waits):
            moved = False
            for k, w in enumerate(waits):
                while w is not None and w[0].passes(w[1] & 1):
                    if w[0].phase <= w[1]:
                        self.early.append(w[2])
                    w = waits[k] = next(threads[k], None)
                    moved = True
            if not moved:
                if not self.landing:
                    return False  # every thread waits: dead
                self.landing.pop().arrive()
        return True


def check(slots, blocks, segments, known=True):
    """The waits that pass too early, over every copy held back."""
    bad, held = set(), -1
    while True:
        m = Model(slots, blocks, segments, held, known)
        done = m.run()
        if m.early:
            bad.update(m.early)
        else:
            assert done, (slots, blocks, segments, held)
        held += 1
        if held >= m.copies:
            return bad


def runs(c):
    """Segments of one to nine tiles, alone and one after another."""
    for n in range(1, 10):
        yield [(n, c, {n - 1})]
    for a in range(1, 8):
        for b in range(1, 8):
            yield [(a, c, {a - 1}), (b, c, {b - 1}), (a, 0, set(range(a))), (b, c, set())]


@pytest.mark.parametrize("blocks,slots", [(1, 6), (2, 5), (1, 10), (2, 10)])
@pytest.mark.parametrize("c", [0, 1, 2])
def test_no_wait_passes_before_its_phase(blocks, slots, c):
    for segments in runs(c):
        assert not check(slots, blocks, segments), segments


def test_a_slot_of_the_other_thread_needs_its_release():
    """Six slots, one row block and one slot of C': tile t's K lies where V of tile t - 3 was, the other thread's.
    Without the wait for that slot's release S would be made from what the slot held; nowhere else is it needed."""
    for blocks, slots in [(1, 6), (2, 5), (1, 10), (2, 10)]:
        for c in (0, 1, 2):
            bad = set().union(*(check(slots, blocks, s, known=False) for s in runs(c)))
            assert bool(bad) == ((blocks, slots, c) == (1, 6, 1)), (blocks, slots, c, bad)
            assert all(re.match("K|V|P|S|Q|C|O|turn|empty|last|slot|sync", x) for x in bad)


def test_the_kernel_has_that_wait_and_these_rings():
    assert re.search(r"ring_slots\(int D, int blocks\) \{ return D == 128 \? \(blocks == 2 \? 5 : 6\) : 10; \}", SOURCE)
    # the release of the slot's use before, then K
    assert re.search(r"BLOCKS == 1 && s\.c_slots == 1 && seq \+ s\.slot\(t\) >= NS\)\s*ok = pwait\(&sh\.empty\[ni\], nph \^ 1, sh, a\);"
                     r"\s*ok = ok && pwait\(&sh\.full\[ni\], nph, sh, a\);", SOURCE)
