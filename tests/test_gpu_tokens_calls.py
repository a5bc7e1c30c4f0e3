"""Calls of the token operators that their documentation allows and that went wrong, or were held right by time alone, once.
Tolerances as in test_gpu_tokens."""
import math

import pytest
import torch

import paper_2502_01277_b200 as octo
from test_gpu_tokens import BF16, F16, F32, _attend_ref, _gen, _ints, _qkv, _u

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_tiles_with_and_without_rows_in_their_second_half(dim):
    """A CTA walks over tiles of 256 rows, each followed by four of 20 rows that have nothing in their second half: the
    record of a full tile stays until the second half has read it, however fast the short ones are through."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = ([256] * sms + [20] * (4 * sms)) * 2
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    n = len(rows)
    q, k, v = _qkv(dim, starts[-1], 3 * n, 1, 1, dim, BF16)
    kw = dict(q_offsets=_ints(starts), k_rows=3, max_q=256)
    want, size, _, _ = _attend_ref(q, k, v, n, **kw)
    tol = (2 * _u(BF16) + 2.0**-15) * size
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = octo.cross_attention(q, k, v, n, status=status, **kw)
    assert ((first.double() - want).abs() <= tol + 1e-30).all()
    for _ in range(100):
        assert torch.equal(octo.cross_attention(q, k, v, n, status=status, **kw), first)
    assert int(status) == 0


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("ilv", [False, True])
@pytest.mark.parametrize("dim,pairs", [(64, 16), (64, 24), (72, 20), (80, 33), (36, 9), (64, 0), (8, 1)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_an_element_that_does_not_turn_stays_alone(dtype, ilv, dim, pairs, bad):
    """Elements behind the rotated ones, and pairs of an axis that is not there, are what they were without a norm: an
    infinity or a NaN among them reaches no other element."""
    g = _gen(dim + pairs)
    rows = 6
    q = torch.randn((rows, 2, dim), generator=g, device="cuda").to(dtype)
    pos = torch.rand((rows, 1), generator=g, device="cuda") * 9
    freqs, axes = torch.rand(pairs, generator=g, device="cuda"), torch.zeros(pairs, dtype=torch.int32, device="cuda")
    if pairs > 2:
        axes[1], axes[2] = -1, 1
    still = list(range(2 * pairs, dim))
    for i in (1, 2) if pairs > 2 else ():
        still += (2 * i, 2 * i + 1) if ilv else (i, i + pairs)
    clean, _ = octo.norm_rotate(q, None, pos, freqs, axes, interleaved=ilv)
    assert torch.equal(clean[..., still], q[..., still])
    for e in still:
        x = q.clone()
        x[1, 0, e] = bad
        out, _ = octo.norm_rotate(x, None, pos, freqs, axes, interleaved=ilv)
        want = clean.clone()
        want[1, 0, e] = bad
        assert torch.equal(out.nan_to_num(nan=777.0), want.nan_to_num(nan=777.0)), e

