"""The attention kernels' forms on the range-checked build (see test_gpu_checked_build): each comparison requires a status
word without any bit."""
import pytest
import torch

import test_gpu_tokens_calls as calls
import test_gpu_tokens_forms as cases
from test_gpu_checked_build import checked  # noqa: F401  (a fixture)
from test_gpu_tokens_forms import forms  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,n,q_rows", [(64, 6, 700), (72, 2, 1000), (128, 1, 1700)])
@pytest.mark.parametrize("masked", [False, True])
def test_row_maxima(checked, forms, dim, n, q_rows, masked):  # noqa: F811
    cases.test_tiles_row_maxima(forms, torch.float16, dim, n, q_rows, masked)


@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 8), (6, 2, 80), (32, 8, 128)])
@pytest.mark.parametrize("q_rows,k_rows", [(17, 1), (49, 64), (130, 257), (300, 450)])
def test_uniform(checked, forms, heads, kv, dim, q_rows, k_rows):  # noqa: F811
    cases.test_tiles_uniform(forms, torch.bfloat16, heads, kv, dim, q_rows, k_rows)


@pytest.mark.parametrize("dim", [64, 128])
def test_windows_and_bounds(checked, forms, dim):  # noqa: F811
    cases.test_tiles_windows_and_bounds(forms, dim)


@pytest.mark.parametrize("n,q_rows,k_rows,heads,kv", [(1, 700, 8192, 1, 1), (3, 130, 9001, 4, 2)])
def test_split_over_the_keys(checked, forms, n, q_rows, k_rows, heads, kv):  # noqa: F811
    cases.test_tiles_split_over_the_keys(forms, torch.bfloat16, n, q_rows, k_rows, heads, kv)


def test_without_any_key(checked, forms):  # noqa: F811
    cases.test_tiles_without_any_key(forms, 20000)


def test_crops_of_a_stage(checked, forms):  # noqa: F811
    cases.test_crops_of_a_stage_in_tiles(forms)


@pytest.mark.parametrize("dim", [64, 128])
def test_tiles_with_and_without_rows_in_their_second_half(checked, dim):  # noqa: F811
    calls.test_attention_tiles_with_and_without_rows_in_their_second_half(dim)
