"""Registers and LDS of the kernels for caches of codes and for drafts, as the compiler's metadata in the library's gfx950 code objects gives them: what decides how
many workgroups a compute unit holds.  No GPU needed."""
from tests.test_chunk_resources import _named, kernels  # noqa: F401

LDS = 160 * 1024


def test_single_tokens_keep_two_workgroups_a_compute_unit(kernels):  # noqa: F811
    for name, k in _named(kernels, r"coded_token_kernelILi(64ELi[01]|128ELi0)E", 6).items():
        assert k["vgpr_count"] <= 128 and k["vgpr_spill_count"] == 0 and 2 * k["group_segment_fixed_size"] <= LDS, name
    for name, k in _named(kernels, r"coded_token_kernelILi128ELi1E", 2).items():  # (shaped: one)
        assert k["vgpr_count"] <= 256 and k["vgpr_spill_count"] == 0 and k["group_segment_fixed_size"] <= LDS, name
    for name, k in _named(kernels, r"coded_token_scores_kernelILi(64|128)E", 8).items():
        assert k["vgpr_count"] <= 128 and k["vgpr_spill_count"] == 0, name


def test_many_rows_keep_three_workgroups_or_groups_a_compute_unit(kernels):  # noqa: F811
    for name, k in _named(kernels, r"(tree_attend_kernelILi128E|coded_attend_kernelILi128E)", 5).items():
        assert k["vgpr_count"] <= 168 and k["vgpr_spill_count"] <= 8 and 3 * k["group_segment_fixed_size"] <= LDS, name
    for name, k in _named(kernels, r"forms_attend_groups_kernelILi128E", 5).items():
        assert k["vgpr_count"] <= 168 and k["vgpr_spill_count"] <= 8 and k["group_segment_fixed_size"] <= LDS, name
    for name, k in _named(kernels, r"(tree_attend_kernel|coded_attend_kernel|forms_attend_groups_kernel)ILi64E", 10).items():
        assert k["vgpr_count"] <= 128 and k["vgpr_spill_count"] == 0, name


def test_few_rows(kernels):  # noqa: F811
    for name, k in _named(kernels, r"forms_attend_few_kernelILi128E", 7).items():
        assert k["vgpr_count"] <= 256 and k["vgpr_spill_count"] == 0 and k["group_segment_fixed_size"] <= LDS, name
    for name, k in _named(kernels, r"forms_attend_few_kernelILi64ELi[02]E", 5).items():  # (two workgroups a compute unit)
        assert k["vgpr_count"] <= 128 and k["vgpr_spill_count"] <= 4 and 2 * k["group_segment_fixed_size"] <= LDS, name


def test_scores_keep_three_workgroups_a_compute_unit(kernels):  # noqa: F811
    for name, k in _named(kernels, r"coded_scores_kernelILi(64|128)E", 12).items():
        assert k["vgpr_count"] <= 168 and k["vgpr_spill_count"] <= 2 and 3 * k["group_segment_fixed_size"] <= LDS, name
    for name, k in _named(kernels, r"coded_scores_few_kernelILi(64|128)E", 12).items():
        assert k["vgpr_count"] <= 256 and k["vgpr_spill_count"] == 0, name


def test_half_of_the_rows_keep_two_waves_a_vector_unit(kernels):  # noqa: F811
    for name, k in _named(kernels, r"forms_attend_half_kernel", 10).items():
        assert k["vgpr_count"] <= 256 and k["vgpr_spill_count"] == 0 and k["group_segment_fixed_size"] <= LDS, name
