"""The compiler's report on the kernels of drafted trees, latents and expanded attention: what lies in scratch memory, and the residency
their launch shapes count on."""
import json
import os

from paper_2405_12591_amd import build as B


def _resources():
    if not os.path.exists(B.RESOURCES_PATH):
        B.build_library()
    with open(B.RESOURCES_PATH) as f:
        return json.load(f)


def test_no_scratch_and_the_residency_that_launches_count_on():
    kinds = {"latent_append_kernel": 8, "latent_read_kernel": 2, "latent_attn_kernel": 12, "latent_narrow_kernel": 4, "latent_join_kernel": 16,
             "tree_attn_kernel": 24, "tree_join_kernel": 12, "expanded_attn_kernel": 4, "expanded_join_kernel": 4}
    seen = dict.fromkeys(kinds, 0)
    for name, r in _resources().items():
        for k in kinds:
            if k not in name:
                continue
            seen[k] += 1
            registers = r["VGPRs"] + r["AGPRs"]
            if k == "latent_attn_kernel" and "Li512ELi4E" in name:
                assert r["ScratchSize"] <= 32, (name, r)         # a few values of a unit, outside the loop over tiles
            else:
                assert r["ScratchSize"] == 0 and r["VGPRs Spill"] == 0, (name, r)
            if k == "tree_attn_kernel":                          # two workgroups a compute unit
                assert registers <= 256 and r["LDS Size"] <= 80 * 1024, (name, r)
            elif k == "expanded_attn_kernel":                    # two of 128 channels, three of 64
                assert registers <= (256 if "Li128E" in name else 170) and r["LDS Size"] <= (80 if "Li128E" in name else 53) * 1024, (name, r)
            elif k == "latent_attn_kernel":                      # one of up to eight waves
                assert registers <= 256 and r["LDS Size"] <= 160 * 1024, (name, r)
            elif k == "latent_narrow_kernel":                    # one of four
                assert registers <= 512 and r["LDS Size"] <= 160 * 1024, (name, r)
    assert seen == kinds
