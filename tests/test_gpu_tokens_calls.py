"""Calls of the token operators that their documentation allows and that went wrong, or were held right by time alone, once.
Tolerances as in test_gpu_tokens."""
import pytest
import torch

import paper_2502_01277_b200 as octo
from test_gpu_tokens import BF16, _attend_ref, _ints, _qkv, _u

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
