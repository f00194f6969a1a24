"""Barriers that the two CTAs of a pair share.  An arrival without a scope holds for its own CTA only, so what it stands for
is not ordered before the other CTA's wait: arrivals on cluster addresses and the waits for them name the cluster."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_36959_b200", "csrc")


def test_barriers_of_a_pair_name_their_scope():
    arrivals = waits = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"mbarrier\.arrive[\w.:]*", text):
            if "shared::cluster" in m.group(0):
                arrivals += 1
                assert ".release.cluster" in m.group(0) or ".relaxed.cluster" in m.group(0), (os.path.basename(path), m.group(0))
        if "barrier_arrive_cluster" in text and "__device__" in text and "mbarrier.try_wait" in text:
            for m in re.finditer(r"mbarrier\.try_wait[\w.:]*", text):
                waits += 1
                assert ".acquire.cluster" in m.group(0), (os.path.basename(path), m.group(0))
    assert arrivals and waits
