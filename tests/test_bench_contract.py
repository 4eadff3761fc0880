"""The benchmark's measured HBM traffic belongs to the sources it was taken on."""
import os
import re

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_traffic_belongs_to_the_headline_sources():
    """A change to one of these sources asks for a new counter run: without it the bench line has no traffic."""
    assert bench.kernel_hash() == bench.TRAFFIC["kernel_hash"]


def test_profile_names_the_same_sources():
    with open(os.path.join(ROOT, "profiles", "postnorm_bert_base_bf16.md")) as f:
        named = re.search(r"Kernel sources hash.*?`([0-9a-f]{16})`", f.read(), re.S)
    assert named and named.group(1) == bench.TRAFFIC["kernel_hash"]
