"""The selection's rows kernel as a protocol (CPU): the warps of a block, the fill count of their list and the block's
barriers, for one chunk, with the warps held back in every order.

All threads have to decide alike whether a chunk's keys may pass the buffer, since one side has barriers of its own.
Behind the barrier that counts the threads that want something a fast warp adds keys, so a fill count that is read there
depends on which warp reads it."""
import itertools
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_2606_01563_gb300", "csrc", "beam_select.cu")).read()
WARPS, VEC, MAX_OUT = 4, 16, 64
BUFFER = MAX_OUT * VEC + 2 * MAX_OUT


class Block:
    """A chunk: the fill count that it finds, and of every warp the threads that want something and the keys they add."""

    def __init__(self, fill, wants, keys, out, early):
        self.fill, self.wants, self.keys, self.out, self.early = fill, sum(wants), keys, out, early

    def warp(self, w):
        fill = self.fill  # (before the barrier)
        yield "count"
        if not self.early:
            fill = self.fill
        if fill + self.wants * VEC > BUFFER:
            if (fill if self.early else self.fill) > self.out:
                yield from ("keep 1", "keep 2", "keep 3")
            yield from ("tops 1", "tops 2")
        self.fill += self.keys[w]
        yield "added"
        if self.fill > 2 * self.out:
            yield from ("keep 1", "keep 2", "keep 3")
        yield "end"

    def run(self, order):
        """The barriers at which the warps met other ones, with the first of `order` always ahead."""
        warps = [self.warp(w) for w in range(WARPS)]
        while True:
            at = {w: next(warps[w], None) for w in order}  # (each as far as its next barrier, one after another)
            if len(set(at.values())) > 1:
                return set(at.values())
            if None in at.values():
                return set()


def mismatches(early, fill, wants, keys, out):
    bad = set()
    for order in itertools.permutations(range(WARPS)):
        bad |= Block(fill, wants, keys, out, early).run(order)
    return bad


CASES = [(0, (32, 32, n - 64, 0), 8, 64) for n in range(65, 73)]   # a first chunk that is a vector of 16 bytes in 65 to 72 threads
CASES += [(0, (32, 32, n - 64, 0), 1, 64) for n in range(68, 73)]  # or one key in each
CASES += [(90, (16, 16, 16, 16), 2, 64), (90, (17, 16, 16, 17), 1, 64), (64, (20, 16, 16, 16), 1, 33)]


@pytest.mark.parametrize("fill,wants,each,out", CASES)
def test_a_count_read_behind_the_barrier_parts_the_warps(fill, wants, each, out):
    assert mismatches(False, fill, wants, [each * n for n in wants], out)


@pytest.mark.parametrize("out", [1, 5, 16, 32, 33, 48, 63, 64])
def test_a_count_read_before_it_does_not(out):
    for fill in range(0, 2 * out + 1, max(1, out // 4)):
        for wants in ((0, 0, 0, 1), (32, 32, 1, 0), (8, 24, 16, 20), (32, 32, 32, 32)):
            for each in (1, 3, VEC):
                assert not mismatches(True, fill, wants, [each * n for n in wants], out)


def test_the_kernel_reads_it_before():
    body = SOURCE[SOURCE.index("beam_rows_kernel(const"):]
    step = body[body.index("const bool any ="):body.index("if (any) {")]
    before, behind = step.split("__syncthreads_count(any)")
    assert "const int fill = sh.fill;" in before
    assert re.search(r"if \(fill \+ wanted \* kVec > kBuffer\) \{\s*if \(fill > a\.out\) keep_best", behind)
    assert "sh.fill" not in behind
    for name, value in (("kThreads = 128, kWarps = kThreads / 32", WARPS), ("kVec = 16", VEC),
                        ("kBuffer = kMaxOut * kVec + 2 * kMaxOut", BUFFER)):
        assert name in SOURCE, (name, value)
