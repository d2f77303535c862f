"""The benchmark's record of HBM traffic is that of the kernel sources it ships with."""
import os

import bench


def test_traffic_record_is_of_these_sources():
    """A change of the attention kernel's code needs new counter runs (the profile has the commands):
    until then the benchmark reports no traffic."""
    assert bench.ATTN_TRAFFIC["sources_sha256"] == bench.attn_sources_digest()


def test_traffic_record_is_that_of_its_profile():
    r = bench.ATTN_TRAFFIC
    text = open(os.path.join(bench.ROOT, r["profile"]), encoding="utf-8").read()
    assert f"{r['bytes_per_launch']:,}" in text and f"{r['nodes_per_launch']:,} attended nodes" in text
    assert r["sources_sha256"][:8] in text
