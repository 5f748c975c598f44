"""Hand-overs between the warps of the ragged products that no run can show to be right: a model of them under random schedules, and the
orderings in the kernels' source."""
import os
import random
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08133_b200", "csrc")


class Barrier:
    """An mbarrier: arrivals and bytes of a phase; a wait by parity passes when the phase of that parity is behind."""

    def __init__(self):
        self.pending, self.bytes, self.phase = 1, 0, 0

    def _check(self):
        if self.pending == 0 and self.bytes == 0:
            self.phase, self.pending = self.phase + 1, 1

    def arrive(self, expect=0):
        assert self.pending == 1
        self.pending, self.bytes = 0, self.bytes + expect
        self._check()

    def land(self):
        self.bytes -= 1
        self._check()

    def passed(self, parity):
        return (self.phase & 1) != parity


def _run(tiles, stages, seed, follow_empty):
    """The loading warp, the warp that fills ragged stages, the issuer, and the loads' arrival, each at its own pace.  False: a product saw
    another block's rows, or somebody waits for ever."""
    rnd = random.Random(seed)
    full, empty, ragged = ([Barrier() for _ in range(stages)] for _ in range(3))
    blocks = [b == n - 1 and r for n, r in tiles for b in range(n)]
    holds, flying, done = [None] * stages, [], []

    def fill(s, k):
        full[s].arrive(1)
        flying.append((s, k))

    def loader():
        for k, is_ragged in enumerate(blocks):
            s, ph = k % stages, k // stages & 1
            while not empty[s].passed(ph ^ 1):
                yield
            if not is_ragged:
                fill(s, k)
            elif not follow_empty:
                ragged[s].arrive()
            yield

    def ragged_loader():
        used = 0
        for k, is_ragged in enumerate(blocks):
            if is_ragged:
                s = k % stages
                while not (empty[s].passed(k // stages & 1 ^ 1) if follow_empty else ragged[s].passed(used >> s & 1)):
                    yield
                used ^= 1 << s
                fill(s, k)
                yield

    def issuer():
        for k in range(len(blocks)):
            s = k % stages
            while not full[s].passed(k // stages & 1):
                yield
            assert holds[s] == k
            done.append(k)
            yield
            empty[s].arrive()
            yield

    roles, pace = [loader(), ragged_loader(), issuer()], [rnd.random() ** 3 + 0.01 for _ in range(4)]
    try:
        for _ in range(200000):
            j = rnd.choices(range(4), pace)[0]
            if j == 3 and flying:
                s, k = flying.pop(rnd.randrange(len(flying)))
                holds[s] = k
                full[s].land()
            elif j < 3 and roles[j] is not None:
                try:
                    next(roles[j])
                except StopIteration:
                    roles[j] = None
            if roles == [None] * 3 and not flying:
                break
    except AssertionError:
        return False
    return len(done) == len(blocks)


@pytest.mark.parametrize("stages", [4, 5, 6])
def test_ragged_stages_are_filled_in_their_turn(stages):
    """A wait by parity must not be a phase ahead: following `empty` past the stages of whole blocks goes wrong, `ragged` does not."""
    wrong = 0
    for seed in range(60):
        r = random.Random(1000 * stages + seed)
        tiles = [(r.choice([1, 1, 2, 3, 8, 18]), r.random() < 0.7) for _ in range(r.randint(1, 30))]
        assert _run(tiles, stages, seed, follow_empty=False)
        wrong += not _run(tiles, stages, seed, follow_empty=True)
    assert wrong > 30


def _source():
    with open(os.path.join(CSRC, "grouped.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_the_ragged_loader_waits_for_its_own_barrier():
    src = _source()
    body = src[src.index("weights_kernel("):]
    body = body[body.index("else if (warp == 2)"):body.index("else if (warp >= 4)")]
    assert "ctl.ragged[s]" in body and "ctl.empty" not in body


def test_a_launch_that_starts_early_ends_late():
    """Whoever waits for a launch may rely on everything ahead of it: each waits for its predecessor before it ends, and lets its follower
    start only after its own wait, where it has one."""
    src = _source()
    close = src[src.index("DEV void close()"):]
    assert close.index("pdl_wait();") < close.index("__syncthreads();")
    start = src[src.index("DEV void open("):]
    assert start.index("if (start == GroupedStart::kAfterLast) pdl_wait();") < start.index("pdl_launch_dependents();")
    rows = src[src.index("list_rows_kernel("):]
    assert rows.index("pdl_wait();") < rows.index("pdl_launch_dependents();") < rows.index("for (")
