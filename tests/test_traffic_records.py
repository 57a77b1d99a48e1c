"""The records of the HBM bytes of an attention launch (profiles/traffic_attn_fwd_*.json) are those of the present source:
bench.py reports none for another."""
import glob
import json
import os

import pytest

import bench

RECORDS = sorted(glob.glob(os.path.join(bench.ROOT, "profiles", "traffic_attn_fwd_*.json")))


def test_there_are_records():
    assert len(RECORDS) >= 6


@pytest.mark.parametrize("path", RECORDS, ids=[os.path.basename(p)[17:-5] for p in RECORDS])
def test_record_is_of_this_source(path):
    with open(path) as f:
        rec = json.load(f)
    digest = bench.src_digest("attn_core.h", "attn.hip")
    assert rec["src_digest"] == digest
    got = bench.traffic_from_profile("attn_fwd", rec["workload"], digest, 0.0)
    assert got == rec["hbm_bytes_per_launch"] > 0
    with open(os.path.join(bench.ROOT, rec["source"])) as f:
        assert digest in f.read()
