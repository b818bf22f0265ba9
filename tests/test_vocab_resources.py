"""The kernels of the embedding, verified drafts and distillation keep everything in registers
(the compiler's report for gfx950; CPU only), as tests/test_kernel_resources.py holds for the
others."""

import pytest

from test_kernel_resources import _kernels, pytestmark  # noqa: F401


@pytest.mark.parametrize("src,kernel", [
    ("embed.hip", "embed_kernel"), ("embed.hip", "rank_kernel"),
    ("embed.hip", "sort_count_kernel"), ("embed.hip", "sort_scatter_kernel"),
    ("embed.hip", "few_kernel"), ("embed.hip", "run_sum_kernel"), ("embed.hip", "run_join_kernel"),
    ("verify.hip", "stats_kernel"), ("verify.hip", "rough_kernel"), ("verify.hip", "exact_kernel"),
    ("verify.hip", "finish_kernel"),
    ("distill.hip", "distill_row_kernel"), ("distill.hip", "distill_part_kernel"),
    ("distill.hip", "distill_join_kernel"), ("distill.hip", "distill_sum_kernel"),
])
def test_no_kernel_spills(src, kernel):
    for _, scratch in _kernels(src, kernel):
        assert scratch == 0, f"{kernel} spills {scratch} bytes per lane"
