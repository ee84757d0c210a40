"""Registers, scratch and LDS of the kernels over a cache in 4 bits and of the verification, from the built library's metadata (no GPU)."""
import re

import test_kernel_resources as resources


def found(pattern):
    return {n: k for n, k in resources.kernels().items() if re.search(pattern, n)}


def test_nothing_is_kept_in_scratch():
    all_of = found("_q4_|AttendQ4Params|verify_")
    assert len(all_of) >= 60
    for n, k in all_of.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n


def test_two_wavefronts_a_simd_of_the_attention():
    """... but for fp32 heads wider than 128: 256 of a SIMD's 512 registers, and half of a CU's LDS"""
    kernels = found("attend_q4_kernel|attend_q4_few_kernel|attend_tile_kernel.*TileQ4")
    assert len(kernels) == 24 + 4 + 7
    for n, k in kernels.items():
        one = "attend_q4_kernelILb1ELi256E" in n
        assert k[".vgpr_count"] <= (512 if one else 256), n
        if "few" not in n and "tile" not in n:
            assert k[".group_segment_fixed_size"] <= 80 * 1024, n


def test_appends_and_reads_fill_a_simd():
    """eight wavefronts a SIMD: 64 registers"""
    kernels = found("kv_append_q4_kernel|kv_read_q4_kernel")
    assert len(kernels) == 16 + 2
    for n, k in kernels.items():
        assert k[".vgpr_count"] <= 64 and k[".group_segment_fixed_size"] == 0, n


def test_verification_of_sixteen_wavefronts_fits():
    (name, k), = found("verify_alone_kernel").items()
    assert k[".vgpr_count"] <= 128 and k[".max_flat_workgroup_size"] == 1024
