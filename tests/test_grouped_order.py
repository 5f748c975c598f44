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


class Count:
    """An mbarrier of `count` arrivals a phase."""

    def __init__(self, count):
        self.count, self.pending, self.phase = count, count, 0

    def arrive(self):
        assert self.pending > 0
        self.pending -= 1
        if self.pending == 0:
            self.phase, self.pending = self.phase + 1, self.count

    def passed(self, parity):
        return (self.phase & 1) != parity


def _share(parts, warps, tiles, seed, wait_free):
    """The warps of results of a cluster that join their partial sums, each at its own pace.  False: a warp read another tile's sums, or somebody
    waits for ever."""
    rnd = random.Random(seed)
    full, free = [Count(parts * warps) for _ in range(parts)], [Count(parts * warps) for _ in range(parts)]
    sums = [[None] * warps for _ in range(parts)]
    wrong = []

    def warp(cta, w):
        for n in range(tiles):
            while wait_free and not free[cta].passed(n & 1 ^ 1):
                yield
            sums[cta][w] = n
            yield
            for c in range(parts):
                full[c].arrive()
            yield
            while not full[cta].passed(n & 1):
                yield
            for c in range(parts):
                wrong.extend(v for v in sums[c] if v != n)
                yield
            for c in range(parts):
                free[c].arrive()
            yield

    running = [warp(c, w) for c in range(parts) for w in range(warps)]
    pace = [rnd.choice([1, 1, 5, 25]) for _ in running]
    for _ in range(60000 * parts):
        if not running:
            return not wrong
        i = rnd.choices(range(len(running)), weights=pace)[0]
        try:
            next(running[i])
        except StopIteration:
            del running[i], pace[i]
        except AssertionError:
            return False
    return False


@pytest.mark.parametrize("parts", [2, 4, 8])
def test_partial_sums_are_read_before_they_are_written_again(parts):
    """A cluster's `part_full` and `part_free`: right under every schedule, wrong without the wait for those that still read."""
    assert all(_share(parts, 3, 6, seed, True) for seed in range(12))
    assert not all(_share(parts, 3, 6, seed, False) for seed in range(12))


def test_partial_sums_are_handed_over_in_order():
    src = _source()
    write = src[src.index("DEV bool write("):src.index("DEV bool publish(")]
    assert write.index("part_free") < write.index("sums[") and write.rindex("__syncwarp()") > write.rindex("sums[")
    assert "mbar_try_wait_acquire_cluster(&ctl.part_free" in write
    publish = src[src.index("DEV bool publish("):src.index("DEV void joined(")]
    assert publish.index("mbar_arrive_release_cluster") < publish.index("mbar_spin_bounded_warp") < publish.index("mbar_try_wait_acquire_cluster")
    for kernel in ("rows_kernel(", "expert_du_kernel("):
        body = src[src.index("\n" + kernel):]
        body = body[:body.index("\n}\n")]
        assert body.index("f.ready();") < body.index("if (kSplit) cluster_sync_all();") < body.index("PartSums<", body.index("f.ready();"))
        assert body.index("sums.publish(") < body.index("sums.joined(") < body.index("sums.release();")
        assert body.rindex("if (kSplit) cluster_sync_all();") < body.index("f.close();")
    split = src[src.index("\nsplit_weights_kernel("):]
    split = split[:split.index("\n}\n")]
    assert split.index("cluster_sync_all();") < split.index("ld.shared::cluster") < split.rindex("cluster_sync_all();") < split.index("f.close();")
