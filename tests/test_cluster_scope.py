"""Arrivals on another CTA's barrier say that they are for the cluster: by default an arrival is a release to its own CTA
alone, which the other CTA's wait does not pair with (the sources, no GPU)."""
import os
import re

import paper_2608_23048_gb300 as roi

CSRC = os.path.join(os.path.dirname(roi.__file__), "csrc")


def sources():
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            yield name, f.read()


def test_arrivals_across_ctas_are_for_the_cluster():
    found = [(name, m[1]) for name, text in sources() for m in re.finditer(r"mbarrier\.arrive([\w.:]*)\.shared::cluster", text)]
    assert found and all(".release.cluster" in how or ".relaxed.cluster" in how for _, how in found), found


def test_shared_memory_is_released_and_tmem_fenced():
    """A relaxed arrival follows a release of shared memory to the cluster, or gives back TMEM behind its own fence."""
    relaxed, tmem = 0, 0
    for name, text in sources():
        for m in re.finditer(r"mbarrier\.arrive\.relaxed\.cluster", text):
            relaxed += 1
            body = text[text.rindex("__device__", 0, m.start()):m.start()]
            assert "fence.release.sync_restrict::shared::cta.cluster" in body or "mbar_arrive_cluster_tmem(" in body, name
        for m in re.finditer(r"mbar_arrive_cluster_tmem\(free", text):
            tmem += 1
            assert re.search(r"tc_fence_before\(\);\s*__syncwarp\(\);\s*if \(lane == 0\) $", text[:m.start()]), name
    assert relaxed == 2 and tmem == 2
