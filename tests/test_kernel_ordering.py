"""Orderings that no run can show to be missing: read in the kernels' sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_08133_b200", "csrc")


def _source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_masked_v_is_handed_to_the_leader_at_cluster_scope():
    """The V tiles of a CTA pair are written by threads of both CTAs and read by a product that the leader issues: the
    arrivals from the other CTA release, and the leader's wait acquires, at cluster scope.  Without a scope both would
    order within one CTA only."""
    common, adapter = _source("common.cuh"), _source("adapter.cu")
    for helper, form in (("mbar_arrive_release_cluster", "mbarrier.arrive.release.cluster.shared::cluster.b64"),
                         ("mbar_try_wait_acquire_cluster", "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64")):
        body = common[common.index("DEV", common.index(helper) - 20):]
        assert form in body[:body.index("\n}")], helper
    uses = [line.strip() for line in adapter.splitlines() if "ctl.vfull" in line and "mbar_init" not in line]
    waits = [u for u in uses if "wait" in u]
    arrivals = [u for u in uses if "arrive" in u]
    assert len(waits) + len(arrivals) == len(uses) and waits and arrivals
    assert all("mbar_wait_acquire_cluster" in u for u in waits), waits
    for u in arrivals:   # an arrival of the leader's own threads may stay in its CTA
        assert "mbar_arrive_release_cluster" in u or re.match(r"if \(rank == 0\) mbar_arrive\(&ctl\.vfull", u), u
