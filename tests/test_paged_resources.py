"""The compiler's report on the kernels of the norm and rotation and of the paged 8-bit cache: nothing in scratch memory, and
the residency their launch shapes count on."""
import json
import os

from paper_2405_12591_amd import build as B


def _resources():
    if not os.path.exists(B.RESOURCES_PATH):
        B.build_library()
    with open(B.RESOURCES_PATH) as f:
        return json.load(f)


def test_no_scratch_and_the_residency_that_launches_count_on():
    kinds = {"rotate_heads_kernel": 16, "paged_append_kernel": 32, "paged_read_kernel": 16, "paged_decode_kernel": 12, "paged_prompt_kernel": 8}
    seen = dict.fromkeys(kinds, 0)
    for name, r in _resources().items():
        for k in kinds:
            if k not in name:
                continue
            seen[k] += 1
            assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (name, r)
            if k in ("paged_decode_kernel", "paged_prompt_kernel"):      # two workgroups a compute unit
                assert r["VGPRs"] + r["AGPRs"] <= 256 and r["LDS Size"] <= 80 * 1024, (name, r)
            if k == "paged_append_kernel":                               # a workgroup is a page: up to 16 waves
                assert r["VGPRs"] + r["AGPRs"] <= 128 and r["LDS Size"] <= 160 * 1024, (name, r)
    assert seen == kinds
