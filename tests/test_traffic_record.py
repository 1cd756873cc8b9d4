"""The memory traffic that the headline benchmark reports was counted on the attention kernel as it is (profiles/)."""
import json
import os

import bench

RECORD = os.path.join(bench.ROOT, "profiles", "tree_attn_bf16.llava7b_layer.hbm_traffic.md")


def test_the_record_is_of_the_present_kernel():
    with open(RECORD) as f:
        rec, = [json.loads(line[len("RESULT "):]) for line in f if line.startswith("RESULT ")]
    assert rec["kernel_source_sha256_16"] == bench.kernel_source_hash(), "the kernel has changed: count its traffic again"
    assert bench.measured_traffic("llava7b_layer") == rec["bytes_per_launch"] >= rec["algorithmic_bytes_per_launch"]
