"""Refusals and layouts of the token calls (positions, norm with rotation, attention) that need no GPU: arguments are
checked before any CUDA call."""
import ctypes
import math

import pytest
import torch

import paper_2502_01277_b200 as octo
from paper_2502_01277_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    return octo.load_library()


def test_struct_layouts():
    assert ctypes.sizeof(B.Heads) == 24
    assert ctypes.sizeof(B.Rotate) == 10 * 4 + 8 + 4 * 24 + 6 * 8 + 8 + 8
    assert ctypes.sizeof(B.Attend) == 6 * 4 + 2 * 8 + 4 * 24 + 2 * 8 + 6 * 8 + 8 + 8 + 8


def _positions(lib, **over):
    a = dict(device=0, items=64, max_items=1, n_items=None, slot_w=224, slot_h=224, patch=16, keep=0, times=None, frames=1,
             positions=64, visible=None)
    a.update(over)
    return lib.octo_patch_positions(a["device"], a["items"], a["max_items"], a["n_items"], a["slot_w"], a["slot_h"], a["patch"],
                                    a["keep"], a["times"], a["frames"], a["positions"], a["visible"], None)


@pytest.mark.parametrize("over", [
    dict(device=-1), dict(max_items=-1), dict(frames=-1), dict(slot_w=0), dict(slot_h=2049), dict(patch=0), dict(patch=15),
    dict(slot_h=225), dict(keep=2), dict(items=None), dict(positions=None)])
def test_positions_refuses(lib, over):
    assert _positions(lib, **over) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("over", [dict(items=66), dict(positions=65), dict(times=2), dict(n_items=1)])
def test_positions_refuses_misaligned_pointers(lib, over):
    assert _positions(lib, **over) == B.OCTO_E_ALIGNMENT


def test_no_items_is_no_work(lib):
    assert _positions(lib, max_items=0, items=None, positions=None) == B.OCTO_OK


def _rotate(**over):
    a = B.Rotate()
    a.device, a.dtype, a.heads, a.kv_heads, a.head_dim, a.pairs, a.num_axes = 0, B.OCTO_F16, 4, 2, 64, 32, 3
    a.rows, a.eps, a.item_rows = 8, 1e-6, 1
    for h in (a.q, a.k, a.q_out, a.k_out):
        h.d_data, h.row_stride, h.head_stride = 4096, 256, 64
    a.d_positions, a.d_freqs, a.d_axes = 256, 512, 768
    for k, v in over.items():
        if "." in k:
            t, f = k.split(".")
            setattr(getattr(a, t), f, v)
        else:
            setattr(a, k, v)
    return a


@pytest.mark.parametrize("over", [
    {"device": -1}, {"dtype": 3}, {"dtype": -1}, {"heads": -1}, {"kv_heads": -1}, {"heads": 0, "kv_heads": 0},
    {"heads": 16385}, {"head_dim": 0}, {"head_dim": 63}, {"head_dim": 258}, {"pairs": 33}, {"pairs": -1}, {"interleaved": 2},
    {"num_axes": 0}, {"num_axes": 9}, {"positions_are_int": 2}, {"rows": -1}, {"rows": (1 << 31) + 1}, {"eps": -1.0},
    {"eps": math.nan}, {"eps": math.inf}, {"d_positions": None}, {"d_freqs": None}, {"d_axes": None}, {"q.d_data": None},
    {"k_out.d_data": None}, {"d_n_items": 64, "item_rows": 0}])
def test_rotate_refuses(lib, over):
    assert lib.octo_norm_rotate(ctypes.byref(_rotate(**over)), None) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("over", [{"q.d_data": 4097}, {"dtype": B.OCTO_F32, "k.d_data": 4098}, {"d_q_weight": 33},
                                  {"d_positions": 258}, {"d_n_items": 2}])
def test_rotate_refuses_misaligned_pointers(lib, over):
    assert lib.octo_norm_rotate(ctypes.byref(_rotate(**over)), None) == B.OCTO_E_ALIGNMENT


def test_rotate_null_and_empty(lib):
    assert lib.octo_norm_rotate(None, None) == B.OCTO_E_INVALID_ARG
    assert lib.octo_norm_rotate(ctypes.byref(_rotate(rows=0)), None) == B.OCTO_OK


def _attend(**over):
    a = B.Attend()
    a.device, a.dtype, a.segments, a.heads, a.kv_heads, a.head_dim = 0, B.OCTO_BF16, 2, 4, 2, 64
    a.q_total, a.k_total, a.q_rows, a.k_rows, a.scale = 2, 32, 1, 16, 0.125
    for h in (a.q, a.k, a.v, a.out):
        h.d_data, h.row_stride, h.head_stride = 4096, 256, 64
    for k, v in over.items():
        if "." in k:
            t, f = k.split(".")
            setattr(getattr(a, t), f, v)
        else:
            setattr(a, k, v)
    return a


BAD_ATTEND = [
    ({"device": -1}, B.OCTO_E_INVALID_ARG), ({"dtype": B.OCTO_F32}, B.OCTO_E_INVALID_ARG), ({"segments": 0}, B.OCTO_E_INVALID_ARG),
    ({"heads": 0}, B.OCTO_E_INVALID_ARG), ({"kv_heads": 0}, B.OCTO_E_INVALID_ARG), ({"kv_heads": 3}, B.OCTO_E_INVALID_ARG),
    ({"head_dim": 0}, B.OCTO_E_INVALID_ARG), ({"head_dim": 60}, B.OCTO_E_INVALID_ARG), ({"head_dim": 136}, B.OCTO_E_INVALID_ARG),
    ({"q_total": -1}, B.OCTO_E_INVALID_ARG), ({"k_total": (1 << 30) + 1}, B.OCTO_E_INVALID_ARG),
    ({"q_rows": 0}, B.OCTO_E_INVALID_ARG), ({"k_rows": -2}, B.OCTO_E_INVALID_ARG), ({"max_q": -1}, B.OCTO_E_INVALID_ARG),
    ({"q_first": 1 << 40}, B.OCTO_E_INVALID_ARG), ({"scale": math.nan}, B.OCTO_E_INVALID_ARG),
    ({"scale": math.inf}, B.OCTO_E_INVALID_ARG), ({"q_total": 1 << 30}, B.OCTO_E_CAPACITY),
    ({"segments": 4097, "d_q_offsets": 64}, B.OCTO_E_CAPACITY), ({"segments": 4097, "d_k_offsets": 64}, B.OCTO_E_CAPACITY)]


@pytest.mark.parametrize("over,code", BAD_ATTEND)
def test_attention_refuses(lib, over, code):
    a, need = _attend(**over), ctypes.c_int64(7)
    assert lib.octo_cross_attention(ctypes.byref(a), None, 0, None) == code
    assert lib.octo_attend_workspace(ctypes.byref(a), ctypes.byref(need)) == code and need.value == 0


@pytest.mark.parametrize("over,code", [
    ({"q.d_data": None}, B.OCTO_E_INVALID_ARG), ({"out.d_data": None}, B.OCTO_E_INVALID_ARG),
    ({"k.d_data": None}, B.OCTO_E_INVALID_ARG), ({"v.d_data": None}, B.OCTO_E_INVALID_ARG),
    ({"q.d_data": 4104}, B.OCTO_E_ALIGNMENT), ({"k.row_stride": 132}, B.OCTO_E_ALIGNMENT),
    ({"v.head_stride": 65}, B.OCTO_E_ALIGNMENT), ({"out.row_stride": 4}, B.OCTO_E_ALIGNMENT),
    ({"d_q_offsets": 66}, B.OCTO_E_ALIGNMENT), ({"d_status": 2}, B.OCTO_E_ALIGNMENT)])
def test_attention_refuses_pointers(lib, over, code):
    assert lib.octo_cross_attention(ctypes.byref(_attend(**over)), None, 0, None) == code


def test_attention_null_and_empty(lib):
    assert lib.octo_cross_attention(None, None, 0, None) == B.OCTO_E_INVALID_ARG
    assert lib.octo_attend_workspace(ctypes.byref(_attend()), None) == B.OCTO_E_INVALID_ARG
    assert lib.octo_cross_attention(ctypes.byref(_attend(q_total=0)), None, 0, None) == B.OCTO_OK


def test_stage_positions_null(lib):
    assert lib.octo_stage_patch_positions(None, 0, 1, 16, None, None, None, None) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("call", [
    lambda: octo.patch_positions(torch.zeros((1, 8), dtype=torch.int32), (224, 224), 16),
    lambda: octo.norm_rotate(torch.zeros((1, 2, 64)), None, torch.zeros((1, 3)), torch.zeros(32), torch.zeros(32).int()),
    lambda: octo.cross_attention(*(torch.zeros((1, 2, 64), dtype=torch.float16),) * 3, 1)])
def test_host_tensors_are_refused(call):
    with pytest.raises(octo.OctoError) as e:
        call()
    assert e.value.code == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("heads,kv_heads,q_total", [(256, 1, (1 << 23) - 1), (256, 256, (1 << 23) - 1), (1, 1, 1 << 30),
                                                    (2, 1, (1 << 30) - 1)])
def test_attention_refuses_rows_that_32_bits_cannot_number(lib, heads, kv_heads, q_total):
    """Rows of a tile are numbered up to 255 beyond the last."""
    fits = q_total * heads <= (1 << 31) - 512
    need = ctypes.c_int64(7)
    rc = lib.octo_attend_workspace(ctypes.byref(_attend(heads=heads, kv_heads=kv_heads, q_total=q_total)), ctypes.byref(need))
    assert (rc != B.OCTO_E_CAPACITY) == fits and need.value == 0


@pytest.mark.parametrize("items", [(1 << 30) + 1, (1 << 31) - 1])
def test_positions_refuses_more_items_than_its_grid_numbers(lib, items):
    """Items are numbered in 32 bits, up to a CTA's more than there are."""
    assert _positions(lib, max_items=items) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("over", [{"out.row_stride": 0}, {"out.head_stride": 0}])
def test_attention_refuses_an_output_whose_rows_or_heads_coincide(lib, over):
    assert lib.octo_cross_attention(ctypes.byref(_attend(**over)), None, 0, None) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("over", [{"q_out.row_stride": 0}, {"q_out.head_stride": 0}, {"k_out.row_stride": 0}, {"k_out.head_stride": 0}])
def test_rotation_refuses_an_output_whose_rows_or_heads_coincide(lib, over):
    assert lib.octo_norm_rotate(ctypes.byref(_rotate(**over)), None) == B.OCTO_E_INVALID_ARG


def test_strides_of_one_row_or_head_mean_nothing(lib):
    """(Where they are accepted the call goes on to the device, which is missing here or takes a call without work.)"""
    one = {"q_total": 1, "heads": 1, "kv_heads": 1, "out.row_stride": 0, "out.head_stride": 0, "device": 1 << 20}
    assert lib.octo_cross_attention(ctypes.byref(_attend(**one)), None, 0, None) == B.OCTO_E_CUDA
    one = {"rows": 1, "heads": 1, "kv_heads": 1, "q_out.row_stride": 0, "q_out.head_stride": 0, "k_out.row_stride": 0,
           "k_out.head_stride": 0, "device": 1 << 20}
    assert lib.octo_norm_rotate(ctypes.byref(_rotate(**one)), None) == B.OCTO_E_CUDA


@pytest.mark.parametrize("over,code", BAD_ATTEND)
def test_attention_plan_refuses_what_the_call_refuses(lib, over, code):
    tile, splits = ctypes.c_int32(7), ctypes.c_int32(7)
    assert lib.octo_attend_plan(ctypes.byref(_attend(**over)), ctypes.byref(tile), ctypes.byref(splits)) == code
    assert (tile.value, splits.value) == (0, 0)


def test_plans_null_and_empty(lib):
    a, b, c = (ctypes.c_int32(7) for _ in range(3))
    refs = [ctypes.byref(x) for x in (a, b, c)]
    assert lib.octo_attend_plan(None, *refs[:2]) == B.OCTO_E_INVALID_ARG
    assert lib.octo_attend_plan(ctypes.byref(_attend()), None, refs[0]) == B.OCTO_E_INVALID_ARG
    assert lib.octo_attend_plan(ctypes.byref(_attend(q_total=0)), *refs[:2]) == B.OCTO_OK and a.value == b.value == 0
    assert lib.octo_rotate_plan(None, *refs) == B.OCTO_E_INVALID_ARG
    assert lib.octo_rotate_plan(ctypes.byref(_rotate()), None, None, None) == B.OCTO_E_INVALID_ARG
    assert lib.octo_rotate_plan(ctypes.byref(_rotate(head_dim=63)), *refs) == B.OCTO_E_INVALID_ARG
    a.value = b.value = c.value = 7
    assert lib.octo_rotate_plan(ctypes.byref(_rotate(rows=0)), *refs) == B.OCTO_OK and a.value == b.value == c.value == 0


@pytest.mark.parametrize("over", [{"out.row_stride": 56}, {"out.head_stride": 8}, {"out.row_stride": 64, "out.head_stride": 64},
                                  {"out.row_stride": 256, "out.head_stride": 312}])
def test_attention_refuses_an_output_whose_rows_or_heads_overlap(lib, over):
    assert lib.octo_cross_attention(ctypes.byref(_attend(**over)), None, 0, None) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("over", [{"q_out.row_stride": 63}, {"k_out.head_stride": -1}, {"q_out.row_stride": 64, "q_out.head_stride": 100},
                                  {"k_out.row_stride": -64}])
def test_rotation_refuses_an_output_whose_rows_or_heads_overlap(lib, over):
    assert lib.octo_norm_rotate(ctypes.byref(_rotate(**over)), None) == B.OCTO_E_INVALID_ARG


@pytest.mark.parametrize("row,head", [(256, 64), (64, 512), (65, 4096), (-256, 64), (128, -64 * 6)])
def test_outputs_of_any_order_are_taken(lib, row, head):
    """(Accepted: the call goes on to a device that is not there.)"""
    a = _rotate(device=1 << 20, **{"q_out.row_stride": row, "q_out.head_stride": head})
    assert lib.octo_norm_rotate(ctypes.byref(a), None) == B.OCTO_E_CUDA
