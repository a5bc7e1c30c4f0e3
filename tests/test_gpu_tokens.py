"""The token calls on a GPU against plain implementations in 64 bits.

Tolerances.  u = half a step of the output's type (eps / 2).
  positions: evaluated in 64 bits and rounded once, u |x| (the reference is in 64 bits, 1e-12 apart).
  norm_rotate: the mean of squares is off by at most about 20 roundings of 2^-24 (16 to 32 terms a lane, a tree of 5),
    half of that after the square root, the factors, cosine and sine by a few more: 32 * 2^-24 of the sizes that are
    added, then u of the result (and half a subnormal step, 2^-25 in fp16).
  cross_attention: every weight is rounded to the type (u of it) and the result once more (u): with
    A = sum_j w_j |v_j| that is 2 u A; scores in binary32 move a weight by less than 2^-16 for scores up to 2^6, so
    2^-15 A more; a weight below fp16's normal range is off by 2^-25 of the largest: 2^-25 sum_j |v_j|."""
import itertools
import math

import numpy as np
import pytest
import torch

import paper_2502_01277_b200 as octo
from paper_2502_01277_b200 import binding as B

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _u(dtype):
    return torch.finfo(dtype).eps / 2


# ---- positions -----------------------------------------------------------------------------------------------------

def _fit(cw, ch, ow, oh, keep):
    if not keep:
        return ow, oh, 0, 0
    if ow * ch <= oh * cw:
        nw, nh = ow, max(1, (2 * ow * ch + cw) // (2 * cw))
    else:
        nw, nh = max(1, (2 * oh * cw + ch) // (2 * ch)), oh
    return nw, nh, (ow - nw) // 2, (oh - nh) // 2


def _positions_ref(rec, slot, p, keep, times):
    ow, oh = slot
    gw, gh = ow // p, oh // p
    pos = np.zeros((len(rec), gh * gw, 3))
    vis = np.zeros((len(rec), gh * gw), np.uint8)
    for n, (frame, _, x0, y0, x1, y1) in enumerate(rec[:, :6].tolist()):
        if x1 <= x0 or y1 <= y0 or frame < 0 or (times is not None and frame >= len(times)):
            continue
        nw, nh, pl, pt = _fit(x1 - x0, y1 - y0, ow, oh, keep)
        for j, i in itertools.product(range(gh), range(gw)):
            pos[n, j * gw + i] = (0.0 if times is None else times[frame],
                                  y0 + ((2 * j + 1) * p - 2 * pt) * (y1 - y0) / (2 * nh),
                                  x0 + ((2 * i + 1) * p - 2 * pl) * (x1 - x0) / (2 * nw))
            vis[n, j * gw + i] = (j * p < pt + nh and (j + 1) * p > pt and i * p < pl + nw and (i + 1) * p > pl)
    return pos, vis


@pytest.mark.parametrize("slot,patch,keep", [
    ((224, 224), 16, 0), ((224, 224), 16, 1), ((96, 33), 3, 1), ((8, 1), 1, 0), ((256, 64), 64, 1), ((2048, 16), 8, 1),
    ((64, 2048), 64, 0)])
@pytest.mark.parametrize("timed", [False, True])
def test_positions(slot, patch, keep, timed):
    rng = np.random.default_rng(slot[0] + patch + keep)
    n = 37
    rec = np.zeros((n, 8), np.int32)
    rec[:, 0] = rng.integers(0, 5, n)
    rec[:, 2], rec[:, 3] = rng.integers(0, 16000, n), rng.integers(0, 9000, n)
    rec[:, 4], rec[:, 5] = rec[:, 2] + rng.integers(1, 384, n), rec[:, 3] + rng.integers(1, 384, n)
    rec[3, 2:6] = (0, 0, 16384, 16384)
    rec[4, 2:6] = (5, 5, 6, 6)
    rec[5, 2:6] = (0, 0, 16384, 1)
    rec[6, 4] = rec[6, 2]  # an empty rectangle
    rec[7, 0] = -1
    rec[8, 0] = 5          # a frame that has no time
    if not timed:
        rec[8, 0] = 4
    times = (rng.random(5) * 1e5).astype(np.float32) if timed else None
    items = torch.from_numpy(rec).cuda()
    pos, vis = octo.patch_positions(items, slot, patch, keep_aspect=bool(keep),
                                    times=None if times is None else torch.from_numpy(times).cuda())
    want, wvis = _positions_ref(rec, slot, patch, keep, times)
    assert np.array_equal(vis.cpu().numpy(), wvis)
    got = pos.cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= 2.0**-24 * np.abs(want) * (1 + 1e-6) + 1e-9).all()


@pytest.mark.parametrize("packed", [0, 1, 7, 20])
def test_positions_leaves_slots_without_an_item(packed):
    items = torch.zeros((9, 8), dtype=torch.int32, device="cuda")
    items[:, 4:6] = 32
    pos = torch.full((9, 4, 3), -5.0, device="cuda")
    vis = torch.full((9, 4), 77, dtype=torch.uint8, device="cuda")
    n = torch.tensor([packed, 100], dtype=torch.int32, device="cuda")
    octo.patch_positions(items, (16, 16), 8, n_items=n, positions=pos, visible=vis)
    k = min(packed, 9)
    assert (vis[:k] == 1).all() and (vis[k:] == 77).all()
    assert (pos[k:] == -5).all() and (pos[:k] != -5).all()


# ---- norm and rotation ---------------------------------------------------------------------------------------------

def _rotate_ref(x, weight, pos, freqs, axes, eps, ilv):
    """Plain form in 64 bits and the sizes that its rotation adds."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    size = y.abs().clone()
    out, r = y.clone(), freqs.numel()
    for i in range(r):
        m, n = (2 * i, 2 * i + 1) if ilv else (i, i + r)
        axis = int(axes[i])
        if not 0 <= axis < pos.shape[1]:
            continue
        phi = (pos[:, axis].double() * freqs[i].double())[:, None]
        out[..., m] = y[..., m] * phi.cos() - y[..., n] * phi.sin()
        out[..., n] = y[..., n] * phi.cos() + y[..., m] * phi.sin()
        size[..., m] = size[..., n] = y[..., m].abs() + y[..., n].abs()
    return out, size


def _rotate_check(got, want, size, dtype):
    err = (got.double() - want).abs()
    tol = _u(dtype) * want.abs() + 32 * 2.0**-24 * size + (2.0**-25 if dtype == F16 else 0.0)
    assert (err <= tol).all(), float((err / tol.clamp(min=1e-30)).max())


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("ilv", [False, True])
@pytest.mark.parametrize("dim,pairs", [(2, 1), (20, 10), (32, 16), (64, 32), (64, 16), (72, 24), (80, 40), (96, 48), (128, 64),
                                       (128, 32), (128, 0), (254, 127), (256, 128), (256, 100)])
def test_rotate(dtype, ilv, dim, pairs):
    g = _gen(dim * 7 + pairs)
    rows, heads, kv = 67, 5, 2
    q = torch.randn((rows, heads, dim), generator=g, device="cuda").to(dtype)
    k = torch.randn((rows, kv, dim), generator=g, device="cuda").to(dtype)
    wq = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(dtype)
    pos = torch.rand((rows, 3), generator=g, device="cuda") * torch.tensor([16777216.0, 1080.0, 1.0], device="cuda")
    freqs = torch.rand(pairs, generator=g, device="cuda") * 2
    axes = torch.randint(0, 3, (pairs,), generator=g, device="cuda").int()
    if pairs > 4:
        axes[1], axes[3] = -1, 3  # no axis of these numbers: the pairs stay
    qo, ko = octo.norm_rotate(q, k, pos, freqs, axes, q_weight=wq, eps=1e-5, interleaved=ilv)
    for got, x, w in ((qo, q, wq), (ko, k, None)):
        want, size = _rotate_ref(x, w, pos, freqs, axes, 1e-5, ilv)
        _rotate_check(got, want, size, dtype)


@pytest.mark.parametrize("dtype,offset", [(F16, 0), (BF16, 1), (F32, 2), (F16, 4), (F32, 0)])
def test_rotate_strides_places_and_integer_positions(dtype, offset):
    """Views of one projection's output at any element offset, outputs of other strides, int32 positions."""
    g = _gen(offset)
    rows, heads, kv, dim = 33, 6, 3, 64
    flat = torch.randn(rows * (heads + 2 * kv) * dim + 64, generator=g, device="cuda").to(dtype)
    qkv = flat[offset:offset + rows * (heads + 2 * kv) * dim].view(rows, heads + 2 * kv, dim)
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv]
    big = torch.full((heads, rows, dim), 9.0, device="cuda", dtype=dtype)
    ko = torch.full((rows, kv, dim + 1), 9.0, device="cuda", dtype=dtype)[..., :dim]
    pos = torch.randint(-(1 << 30), 1 << 30, (rows, 1), generator=g, device="cuda").int()
    freqs, axes = torch.rand(32, generator=g, device="cuda"), torch.zeros(32, device="cuda").int()
    w = torch.randn(dim, generator=g, device="cuda").to(dtype)
    octo.norm_rotate(q, k, pos, freqs, axes, q_weight=w, k_weight=w, out=(big.transpose(0, 1), ko))
    for got, x in ((big.transpose(0, 1), q), (ko, k)):
        want, size = _rotate_ref(x, w, pos, freqs, axes, 1e-6, False)
        _rotate_check(got, want, size, dtype)


def test_rotate_in_place_and_rows_without_an_item():
    g = _gen(3)
    q = torch.randn((40, 3, 64), generator=g, device="cuda").to(BF16)
    before = q.clone()
    pos = torch.rand((40, 2), generator=g, device="cuda") * 100
    freqs, axes = torch.rand(32, generator=g, device="cuda"), torch.arange(32, device="cuda").int() % 2
    n = torch.tensor([5], dtype=torch.int32, device="cuda")
    out, none = octo.norm_rotate(q, None, pos, freqs, axes, n_items=n, item_rows=7, out=(q, None))
    assert out is q and none is None
    want, size = _rotate_ref(before, None, pos, freqs, axes, 1e-6, False)
    _rotate_check(q[:35], want[:35], size[:35], BF16)
    assert torch.equal(q[35:], before[35:])
    for items, left in ((0, 0), (-3, 0), (100, 40)):
        q.copy_(before)
        n.fill_(items)
        octo.norm_rotate(q, None, pos, freqs, axes, n_items=n, item_rows=7, out=(q, None))
        assert torch.equal(q[left:], before[left:]) and (left == 0 or not torch.equal(q, before))


def test_rotate_zero_rows_and_zero_heads_norm():
    q = torch.zeros((2, 1, 64), device="cuda", dtype=F16)
    pos, freqs, axes = torch.ones((2, 1), device="cuda"), torch.ones(32, device="cuda"), torch.zeros(32, device="cuda").int()
    w = torch.ones(64, device="cuda", dtype=F16)
    out, _ = octo.norm_rotate(q, None, pos, freqs, axes, q_weight=w)
    assert (out == 0).all()
    empty, _ = octo.norm_rotate(q[:0], None, pos[:0], freqs, axes)
    assert empty.shape == (0, 1, 64)


# ---- attention -----------------------------------------------------------------------------------------------------

def _bounds(offsets, s, rows, first, total, most):
    b, e = (s, s + 1) if offsets is None else (int(offsets[s]), int(offsets[s + 1]))
    b, e = (min(max((x - first) * rows, 0), total) for x in (b, e))
    return b, b + (min(e - b, most) if most else e - b)


def _attend_ref(q, k, v, n, *, q_offsets=None, k_offsets=None, q_rows=1, k_rows=1, q_first=0, k_first=0, max_q=None, max_k=None,
                key_mask=None, scale=None, out=None):
    """Plain form in 64 bits, the weighted sizes A, the plain sum of sizes, and which rows belong to a segment."""
    want = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    size, plain = torch.zeros_like(want), torch.zeros_like(want)
    rows = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    group, scale = q.shape[1] // k.shape[1], q.shape[2] ** -0.5 if scale is None else scale
    for s in range(n):
        q0, q1 = _bounds(q_offsets, s, q_rows, q_first, q.shape[0], max_q)
        k0, k1 = _bounds(k_offsets, s, k_rows, k_first, k.shape[0], max_k)
        if q1 <= q0:
            continue
        rows[q0:q1] = True
        at = torch.arange(k0, max(k0, k1), device="cuda")
        if key_mask is not None:
            at = at[key_mask[at] != 0]
        if not at.numel():
            continue
        for h in range(q.shape[1]):
            kk, vv = k[at, h // group].double(), v[at, h // group].double()
            w = torch.softmax(q[q0:q1, h].double() @ kk.T * scale, -1)
            want[q0:q1, h], size[q0:q1, h] = w @ vv, w @ vv.abs()
            plain[q0:q1, h] = vv.abs().sum(0)
    return want, size, plain, rows


def _attend_check(q, k, v, n, **kw):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    octo.cross_attention(q, k, v, n, out=out, status=status, **kw)
    want, size, plain, rows = _attend_ref(q, k, v, n, **kw)
    assert int(status) == 0
    assert (out[~rows] == 7).all(), "rows of no segment were written"
    u = _u(q.dtype)
    tol = (2 * u + 2.0**-15) * size + (2.0**-25 * (plain + 1) if q.dtype == F16 else 0.0)
    err = (out.double() - want).abs()[rows]
    assert not torch.isnan(out[rows]).any()
    assert (err <= tol[rows] + 1e-30).all(), float((err / tol[rows].clamp(min=1e-30)).max())
    return out


def _qkv(seed, q_total, k_total, heads, kv, dim, dtype, fused=False, gain=1.5):
    g = _gen(seed)
    q = (gain * torch.randn((q_total, heads, dim), generator=g, device="cuda")).to(dtype)
    if fused:
        both = torch.randn((k_total, 2, kv, dim), generator=g, device="cuda").to(dtype)
        return q, both[:, 0], both[:, 1]
    return (q, torch.randn((k_total, kv, dim), generator=g, device="cuda").to(dtype),
            torch.randn((k_total, kv, dim), generator=g, device="cuda").to(dtype))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 8), (2, 2, 64), (4, 1, 128), (6, 2, 80), (3, 3, 40), (8, 8, 72), (32, 8, 128)])
@pytest.mark.parametrize("q_rows,k_rows", [(1, 1), (1, 15), (1, 64), (3, 65), (1, 197), (16, 129), (17, 128), (49, 1000),
                                           (130, 257)])
def test_attention_uniform(dtype, heads, kv, dim, q_rows, k_rows):
    n = 3
    q, k, v = _qkv(q_rows + k_rows, n * q_rows, n * k_rows, heads, kv, dim, dtype, fused=dim % 16 == 0)
    _attend_check(q, k, v, n, q_rows=q_rows, k_rows=k_rows)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("per_item,dim,heads,kv", [(1, 64, 4, 4), (7, 128, 4, 1), (37, 80, 6, 2), (100, 64, 2, 2)])
@pytest.mark.parametrize("masked", [False, True])
def test_attention_ragged(dtype, per_item, dim, heads, kv, masked):
    """Offsets as the stage writes them: segments without items, segments without keys, slots behind the last item."""
    items, keys = [3, 0, 5, 1, 0, 2], [130, 40, 0, 700, 0, 257]
    qo, ko = [0], [0]
    for a, b in zip(items, keys):
        qo.append(qo[-1] + a)
        ko.append(ko[-1] + b)
    q, k, v = _qkv(per_item, (qo[-1] + 4) * per_item, ko[-1] + 9, heads, kv, dim, dtype)
    mask = (torch.rand(ko[-1] + 9, generator=_gen(1), device="cuda") < 0.6).to(torch.uint8) if masked else None
    if masked:
        mask[ko[5]:] = 0  # the last segment sees nothing
        k[mask == 0], v[mask == 0] = math.nan, math.inf
    k[ko[-1]:], v[ko[-1]:] = math.inf, math.nan  # behind the last segment
    _attend_check(q, k, v, 6, q_offsets=_ints(qo), k_offsets=_ints(ko), q_rows=per_item, key_mask=mask)
    _attend_check(q, k, v, 6, q_offsets=_ints(qo), k_offsets=_ints(ko), q_rows=per_item, key_mask=mask,
                  max_q=max(items) * per_item, max_k=700)


@pytest.mark.parametrize("q_rows", [1, 40])
def test_attention_windows_and_bounds(q_rows):
    """A window of the item list (first), and segments longer than the bounds that the caller gives."""
    qo, ko = [0, 4, 9, 9, 15], [5, 10, 30, 31, 60]
    q, k, v = _qkv(1, 8 * q_rows, 40 * 8, 4, 2, 64, BF16)
    kw = dict(q_offsets=_ints(qo), k_offsets=_ints(ko), q_rows=q_rows, k_rows=8)
    _attend_check(q, k, v, 4, q_first=3, k_first=7, **kw)
    _attend_check(q, k, v, 4, q_first=-1, k_first=20, max_q=2 * q_rows, max_k=33, **kw)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,q_rows,k_rows,heads,kv", [(1, 1, 20000, 8, 1), (2, 2, 9001, 8, 8), (1, 100, 30000, 2, 1),
                                                      (1, 300, 8192, 1, 1)])
def test_attention_long(dtype, n, q_rows, k_rows, heads, kv):
    """Work split over the keys and joined."""
    q, k, v = _qkv(n, n * q_rows, n * k_rows, heads, kv, 128, dtype)
    mask = torch.ones(n * k_rows, dtype=torch.uint8, device="cuda")
    mask[100:5000] = 0
    _attend_check(q, k, v, n, q_rows=q_rows, k_rows=k_rows)
    _attend_check(q, k, v, n, q_rows=q_rows, k_rows=k_rows, key_mask=mask)
    lengths = _ints([0, 300] if n == 1 else [0, 9000, 9000])  # most splits have nothing to do
    _attend_check(q, k, v, n, q_rows=q_rows, k_offsets=lengths)


@pytest.mark.parametrize("q_rows", [1, 64, 300])
def test_attention_row_maxima(q_rows):
    """Scores far apart, growing along the keys, equal, and a negative scale; the running maximum moves a lot."""
    q, k, v = _qkv(5, q_rows, 1500, 2, 2, 64, BF16)
    grow = torch.linspace(-3, 3, 1500, device="cuda")[:, None, None]
    kk = (k.float().abs() * grow).to(BF16)
    qq = q.abs()
    for scale in (0.125, -0.125, 0.0):
        _attend_check(qq, kk, v, 1, q_rows=q_rows, k_rows=1500, scale=scale)
    _attend_check(qq, kk.flip(0), v, 1, q_rows=q_rows, k_rows=1500)
    same = k[:1].expand(1500, -1, -1).contiguous()
    _attend_check(q, same, v, 1, q_rows=q_rows, k_rows=1500)


@pytest.mark.parametrize("q_rows", [1, 200])
def test_attention_visible_nan_and_infinities_come_through(q_rows):
    q, k, v = _qkv(6, q_rows, 600, 1, 1, 64, BF16)
    v[137, 0, 3] = math.nan
    out = octo.cross_attention(q, k, v, 1, q_rows=q_rows, k_rows=600)
    assert torch.isnan(out[:, 0, 3]).all() and not torch.isnan(out[:, 0, :3]).any()
    k2 = k.clone()
    k2[500] = math.nan
    assert torch.isnan(octo.cross_attention(q, k2, v, 1, q_rows=q_rows, k_rows=600)).all()


def test_attention_64_bit_offsets():
    """Keys that lie more than 2^32 elements behind the first."""
    k_total, kv, dim = 1100, 1, 64
    apart = (1 << 32) // 1024
    store = torch.zeros((1 << 32) + 80 * apart, dtype=BF16, device="cuda")
    k = torch.as_strided(store, (k_total, kv, dim), (apart, dim, 1), 0)
    v = torch.as_strided(store, (k_total, kv, dim), (apart, dim, 1), 1024)
    g = _gen(9)
    k.copy_(torch.randn((k_total, kv, dim), generator=g, device="cuda"))
    v.copy_(torch.randn((k_total, kv, dim), generator=g, device="cuda"))
    for q_rows in (1, 140):
        q = torch.randn((q_rows, 2, dim), generator=g, device="cuda").to(BF16)
        _attend_check(q, k, v, 1, q_rows=q_rows, k_rows=k_total)
    del store, k, v
    torch.cuda.empty_cache()


def test_attention_is_repeatable_on_streams_and_in_graphs():
    cases = []
    for seed, (n, qr, kr) in enumerate([(3, 1, 5000), (4, 90, 700), (1, 300, 6000)]):
        q, k, v = _qkv(seed, n * qr, n * kr, 4, 2, 128, BF16)
        want = _attend_check(q, k, v, n, q_rows=qr, k_rows=kr)
        cases.append((q, k, v, n, qr, kr, want))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        for st, (q, k, v, n, qr, kr, want) in zip(streams, cases):
            outs.append((octo.cross_attention(q, k, v, n, q_rows=qr, k_rows=kr, stream=st), want))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in outs)
    graphs = []
    for q, k, v, n, qr, kr, want in cases:
        out, gr = torch.zeros_like(q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            octo.cross_attention(q, k, v, n, q_rows=qr, k_rows=kr, out=out)
        graphs.append((gr, out, want))
    for _ in range(3):
        for (gr, out, _), st in zip(graphs, streams):
            out.zero_()
        torch.cuda.synchronize()
        for (gr, _, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for _, out, want in graphs)


def test_refusals_on_the_gpu():
    q, k, v = _qkv(0, 4, 8, 4, 2, 64, BF16)
    off = _ints([0, 1, 2])
    bad = [
        lambda: octo.cross_attention(q.float(), k, v, 1), lambda: octo.cross_attention(q, k.half(), v, 1),
        lambda: octo.cross_attention(q, k, v[:4], 1), lambda: octo.cross_attention(q[:, :3], k, v, 1),
        lambda: octo.cross_attention(q, k, v, 3, q_offsets=off), lambda: octo.cross_attention(q, k, v, 2, q_offsets=off.long()),
        lambda: octo.cross_attention(q, k, v, 2, q_offsets=off.cpu()),
        lambda: octo.cross_attention(q, k, v, 1, key_mask=torch.ones(7, device="cuda", dtype=torch.uint8)),
        lambda: octo.cross_attention(q, k, v, 1, out=q[:2]), lambda: octo.cross_attention(q, k, v, 0),
        lambda: octo.cross_attention(q[..., ::2], k[..., ::2], v[..., ::2], 1),
        lambda: octo.cross_attention(q[..., :60], k[..., :60], v[..., :60], 1),
        lambda: octo.cross_attention(q[..., 4:60], k[..., 4:60], v[..., 4:60], 1),
        lambda: octo.patch_positions(_ints([[0] * 8]), (224, 224), 15), lambda: octo.patch_positions(_ints([[0] * 7]), (8, 8), 8),
        lambda: octo.norm_rotate(q, k, torch.zeros((4, 1), device="cuda"), torch.zeros(32, device="cuda"), off),
        lambda: octo.norm_rotate(q, k[:2], torch.zeros((4, 1), device="cuda"), torch.zeros(2, device="cuda"), off),
        lambda: octo.norm_rotate(q, None, torch.zeros((4, 1)), torch.zeros(2, device="cuda"), off),
        lambda: octo.norm_rotate(q, None, torch.zeros((4, 1), device="cuda"), torch.zeros(2, device="cuda"), off,
                                 q_weight=torch.ones(64, device="cuda"))]
    for call in bad:
        with pytest.raises(octo.OctoError):
            call()
    assert torch.cuda.current_device() == 0


# ---- together, as behind a stage -----------------------------------------------------------------------------------

def test_crops_attend_to_their_frames():
    """A pass of the stage, then its crops' tokens: positions, norm with rotation, attention to the states of the
    frame each was cut from -- all from the tables the stage left on the device, eagerly and from one captured graph."""
    import workloads
    from gpu_harness import make_stage, upload_frames
    b = workloads.make_batch("two_branch", batch=3)
    wl = b.workload
    st = make_stage(wl, b.n, branches=((224, 224), (64, 32)), crop_options=[None, {"keep_aspect": True}])
    with pytest.raises(octo.OctoError):
        st.patch_positions(0, 8, 16)
    frames, head = upload_frames(b.frames), torch.from_numpy(b.head).cuda()
    heads, kv, dim, patch, cap = 4, 2, 64, 32, 96
    g = _gen(11)
    times = torch.tensor([10.0, 20.0, 30.0], device="cuda")
    # the canvases as items: whole frames, fitted
    canvas = torch.zeros((b.n, 8), dtype=torch.int32)
    for i, (w, h) in enumerate(b.sizes):
        canvas[i, 0], canvas[i, 4], canvas[i, 5] = i, w, h
    canvas = canvas.cuda()
    states = (wl.net_size // patch) ** 2
    freqs = (100.0 ** (-torch.arange(dim // 2, device="cuda").float() / (dim // 2))) * 0.05
    axes = torch.arange(dim // 2, device="cuda").int() % 3
    wq, wk = torch.rand(dim, generator=g, device="cuda").to(F16), torch.rand(dim, generator=g, device="cuda").to(F16)
    k0 = torch.randn((b.n * states, kv, dim), generator=g, device="cuda").to(F16)
    v0 = torch.randn((b.n * states, kv, dim), generator=g, device="cuda").to(F16)

    for branch, side in ((0, 224), (1, 64)):
        tokens = (side // patch) * ((side if branch == 0 else 32) // patch)
        q0 = torch.randn((cap * tokens, heads, dim), generator=g, device="cuda").to(F16)
        out = torch.full_like(q0, 7.0)
        n_items = torch.zeros(2, dtype=torch.int32, device="cuda")
        offsets = torch.zeros(b.n + 1, dtype=torch.int32, device="cuda")
        crops = torch.zeros((cap, 3, side if branch == 0 else 32, side), dtype=F16, device="cuda")
        kept = {}

        def one_pass():
            st.preprocess(frames, b.sizes)
            st.postprocess(head)
            st.crop(branch, cap, out=crops, offsets=offsets, n_items=n_items)
            pos, vis = st.patch_positions(branch, cap, patch, times=times)
            kpos, kvis = octo.patch_positions(canvas, (wl.net_size, wl.net_size), patch, keep_aspect=True, times=times)
            q, _ = octo.norm_rotate(q0, None, pos.view(-1, 3), freqs, axes, q_weight=wq, n_items=n_items, item_rows=tokens)
            k, _ = octo.norm_rotate(k0, None, kpos.view(-1, 3), freqs, axes, q_weight=wk)
            octo.cross_attention(q, k, v0, b.n, q_offsets=offsets, q_rows=tokens, k_rows=states, max_k=states,
                                 key_mask=kvis.view(-1), out=out)
            kept.update(pos=pos, vis=vis, kpos=kpos, kvis=kvis, q=q, k=k)

        one_pass()
        torch.cuda.synchronize()
        packed, off = int(n_items[0]), offsets.tolist()
        assert 0 < packed < cap and off[-1] == packed
        table = st.item_table(branch, packed)
        rec = np.stack([table[f] for f in ("frame", "det", "rx0", "ry0", "rx1", "ry1")], 1)
        slot = (st.cfg.branch[branch].out_w, st.cfg.branch[branch].out_h)
        want, wvis = _positions_ref(rec, slot, patch, branch, times.tolist())
        assert np.array_equal(kept["vis"][:packed].cpu().numpy(), wvis)
        got = kept["pos"][:packed].cpu().numpy().astype(np.float64)
        assert (np.abs(got - want) <= 2.0**-24 * np.abs(want) * (1 + 1e-6) + 1e-9).all()
        rows = packed * tokens
        for got, x, w, pos in ((kept["q"][:rows], q0[:rows], wq, kept["pos"].view(-1, 3)[:rows]),
                               (kept["k"], k0, wk, kept["kpos"].view(-1, 3))):
            ref, size = _rotate_ref(x, w, pos, freqs, axes, 1e-6, False)
            _rotate_check(got, ref, size, F16)
        assert 0 < int(kept["kvis"].sum()) < b.n * states  # wide frames leave canvas
        ref, size, plain, used = _attend_ref(kept["q"], kept["k"], v0, b.n, q_offsets=offsets, q_rows=tokens, k_rows=states,
                                             key_mask=kept["kvis"].view(-1))
        assert int(used.sum()) == rows and (out[rows:] == 7).all()
        err, tol = (out.double() - ref).abs()[:rows], ((2 * _u(F16) + 2.0**-15) * size + 2.0**-25 * (plain + 1))[:rows]
        assert (err <= tol).all()
        eager = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one_pass()
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        with pytest.raises(octo.OctoError):
            st.patch_positions(branch, cap, 5)
    assert st.status() == 0
    st.preprocess(frames, b.sizes)  # a new batch: the old table is not its
    st.postprocess(head)
    with pytest.raises(octo.OctoError) as e:
        st.patch_positions(0, 8, 16)
    assert e.value.code == B.OCTO_E_NO_POSTPROCESS
    st.close()


def _random_case(rng, g):
    """A call with everything drawn: head layout, segments with none or many rows and keys, mask, windows, bounds."""
    kv = rng.choice([1, 2, 4])
    heads, dim, dtype = kv * rng.choice([1, 2, 3, 8]), rng.choice([8, 24, 64, 72, 128]), rng.choice([F16, BF16])
    n, rows, step = rng.randint(1, 30), rng.choice([1, 7, 49, 130]), rng.choice([1, 1, 16])
    qo, ko = [0], [0]
    for _ in range(n):
        qo.append(qo[-1] + rng.choice([0, 1, 3, 9]))
        ko.append(ko[-1] + rng.choice([0, 1, 15, 63, 64, 65, 128, 129, 500]))
    q, k, v = _qkv(rng.randrange(1 << 30), qo[-1] * rows + 3, ko[-1] * step + 1, heads, kv, dim, dtype, fused=rng.random() < 0.5)
    kw = dict(q_offsets=_ints(qo), k_offsets=_ints(ko), q_rows=rows, k_rows=step)
    if rng.random() < 0.5:
        kw["key_mask"] = (torch.rand(k.shape[0], generator=g, device="cuda") < rng.random()).to(torch.uint8)
    if rng.random() < 0.3:
        kw["max_q"], kw["max_k"] = rng.randint(1, 9 * rows), rng.randint(1, 500 * step)
    return q, k, v, n, kw


@pytest.mark.parametrize("seed", range(24))
def test_attention_random_calls(seed):
    import random
    rng, g = random.Random(seed), _gen(seed)
    for _ in range(3):
        q, k, v, n, kw = _random_case(rng, g)
        _attend_check(q, k, v, n, **kw)


def test_attention_many_calls_agree():
    """The same calls over and over, back to back: hand-overs inside the kernel that depended on which of its parts was
    faster showed up as one call among thousands (a wait that ran out, or a record read before it was written)."""
    import random
    rng, g = random.Random(99), _gen(99)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(150):
        q, k, v, n, kw = _random_case(rng, g)
        first = octo.cross_attention(q, k, v, n, out=torch.zeros_like(q), status=status, **kw)
        rest = [octo.cross_attention(q, k, v, n, out=torch.zeros_like(q), status=status, **kw) for _ in range(12)]
        assert all(torch.equal(first, x) for x in rest)
        assert int(status) == 0


@pytest.mark.parametrize("q_rows", [1, 3, 20, 300])
def test_attention_without_any_key(q_rows):
    q, k, v = _qkv(0, 2 * q_rows, 0, 4, 2, 64, BF16)
    out = octo.cross_attention(q, k, v, 2, q_rows=q_rows)
    assert (out == 0).all()
    q, k, v = _qkv(0, 2 * q_rows, 600, 4, 2, 64, BF16)
    k.fill_(math.nan), v.fill_(math.nan)
    out = octo.cross_attention(q, k, v, 2, q_rows=q_rows, k_rows=300, key_mask=torch.zeros(600, dtype=torch.bool, device="cuda"))
    assert (out == 0).all()


def test_attention_no_rows():
    q, k, v = _qkv(0, 0, 10, 4, 2, 64, BF16)
    assert octo.cross_attention(q, k, v, 1, k_rows=10).shape == (0, 4, 64)
    q, k, v = _qkv(0, 5, 10, 4, 2, 64, BF16)
    out = torch.full_like(q, 7.0)
    octo.cross_attention(q, k, v, 3, q_offsets=_ints([0, 0, 0, 0]), k_rows=3, out=out)
    assert (out == 7).all()


def test_attention_one_wide_head_for_many_queries():
    """All heads share one key head; keys and values are the same memory, seen through strides of their own."""
    g = _gen(4)
    base = torch.randn((500, 3, 128), generator=g, device="cuda").to(BF16)
    q = torch.randn((6, 64, 128), generator=g, device="cuda").to(BF16)
    k = base[:, :1]
    _attend_check(q, k, k, 2, q_rows=3, k_rows=250)
    _attend_check(q.transpose(0, 1).contiguous().transpose(0, 1), base[:, 1:2], base[:, 2:], 6, q_rows=1, k_rows=83)


@pytest.mark.parametrize("q_rows,dim", [(3, 64), (140, 64), (60, 128), (300, 128)])
@pytest.mark.parametrize("period,edge", [(1600, 350), (100, 3), (129, 1), (128, 0), (64, 31), (257, 128), (1000, 499)])
def test_attention_banded_masks(q_rows, dim, period, edge):
    """Visible keys in runs (frames between their canvas bands): runs longer and shorter than a tile, single keys between."""
    q, k, v = _qkv(period, 2 * q_rows, 2 * 3333, 2, 1, dim, BF16)
    place = torch.arange(k.shape[0], device="cuda") % period
    mask = ((place >= edge) & (place < period - edge)).to(torch.uint8)
    k[mask == 0], v[mask == 0] = math.nan, math.nan
    _attend_check(q, k, v, 2, q_rows=q_rows, k_rows=3333, key_mask=mask)
    _attend_check(q, k, v, 3, q_rows=q_rows, k_offsets=_ints([5, 6, 3000, 6666]), key_mask=mask)


def test_results_on_another_stream_are_not_taken_from_memory_in_use():
    """What a call on a given stream allocates is that stream's: memory that the current stream has let go of may still
    be written by work under way there."""
    g = _gen(11)
    q, k, v = _qkv(11, 1, 20000, 8, 1, 64, BF16)
    items = torch.zeros((64, 8), dtype=torch.int32, device="cuda")
    items[:, 4:6] = 100
    pos = torch.rand((64, 1), generator=g, device="cuda") * 100
    freqs, axes = torch.rand(32, generator=g, device="cuda"), torch.zeros(32, dtype=torch.int32, device="cuda")
    x = torch.randn((64, 4, 64), generator=g, device="cuda").to(BF16)
    calls = [lambda st: (octo.cross_attention(q, k, v, 1, k_rows=20000, stream=st),),
             lambda st: octo.norm_rotate(x, x[:, :2], pos, freqs, axes, stream=st),
             lambda st: octo.patch_positions(items, (224, 224), 16, stream=st)]
    side = torch.cuda.Stream()
    for call in calls:
        want = call(None)
        torch.cuda.synchronize()
        in_use = [torch.empty_like(w) for w in want for _ in range(3)]
        torch.cuda._sleep(100_000_000)
        for b in in_use:
            b.fill_(77)
        del in_use, b
        got = call(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_attention_rows_half_a_gigabyte_apart():
    """Four rows of such a tensor are 2^31 bytes."""
    apart, k_total, q_rows, dim = (1 << 28) + 8, 128, 34000, 64
    if torch.cuda.mem_get_info()[0] < 2 * apart * k_total + (4 << 30):
        pytest.skip("needs 73 GB of device memory")
    store = torch.empty(apart * k_total, dtype=BF16, device="cuda")
    k = torch.as_strided(store, (k_total, 1, dim), (apart, dim, 1), 0)
    v = torch.as_strided(store, (k_total, 1, dim), (apart, dim, 1), 1024)
    g = _gen(12)
    k.copy_(torch.randn((k_total, 1, dim), generator=g, device="cuda"))
    v.copy_(torch.randn((k_total, 1, dim), generator=g, device="cuda"))
    q = torch.randn((q_rows, 1, dim), generator=g, device="cuda").to(BF16)
    _attend_check(q, k, v, 1, q_rows=q_rows, k_rows=k_total)
    mask = torch.ones(k_total, dtype=torch.uint8, device="cuda")
    mask[7] = 0
    _attend_check(q, k, v, 1, q_rows=q_rows, k_rows=k_total, key_mask=mask)
    del store, k, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("first_item,cap", [(0, 5), (5, 7), (3, 1000), (100000, 8)])
def test_windows_of_a_branch(first_item, cap):
    """Positions of a window of a branch's items, and attention of its tokens (the offsets count all items)."""
    import workloads
    from gpu_harness import make_stage, upload_frames
    b = workloads.make_batch("two_branch", batch=3)
    wl = b.workload
    st = make_stage(wl, b.n, branches=((224, 224), (64, 32)))
    frames, head = upload_frames(b.frames), torch.from_numpy(b.head).cuda()
    st.preprocess(frames, b.sizes)
    st.postprocess(head)
    _, offsets, n_items = st.crop(0, cap, first_item=first_item)
    pos = torch.full((cap, 196, 3), -5.0, device="cuda")
    vis = torch.full((cap, 196), 9, dtype=torch.uint8, device="cuda")
    st.patch_positions(0, cap, 16, positions=pos, visible=vis)
    packed, total = n_items.tolist()
    assert packed == max(0, min(cap, total - first_item)) and total > 12
    table = st.item_table(0, packed) if packed else None
    if packed:
        rec = np.stack([table[f] for f in ("frame", "det", "rx0", "ry0", "rx1", "ry1")], 1)
        want, wvis = _positions_ref(rec, (224, 224), 16, 0, None)
        got = pos[:packed].cpu().numpy().astype(np.float64)
        assert (np.abs(got - want) <= 2.0**-24 * np.abs(want) * (1 + 1e-6) + 1e-9).all()
        assert np.array_equal(vis[:packed].cpu().numpy(), wvis)
    assert (pos[packed:] == -5).all() and (vis[packed:] == 9).all()
    tokens, states = 3, 70
    g = _gen(first_item)
    q = torch.randn((cap * tokens, 4, 64), generator=g, device="cuda").to(BF16)
    k, v = (torch.randn((b.n * states, 2, 64), generator=g, device="cuda").to(BF16) for _ in range(2))
    out = torch.full_like(q, 7.0)
    octo.cross_attention(q, k, v, b.n, q_offsets=offsets, q_rows=tokens, k_rows=states, q_first=first_item, out=out)
    assert (out[packed * tokens:] == 7).all()
    for i in range(packed):  # every item to the states of its own frame
        f = int(table["frame"][i])
        one = slice(i * tokens, (i + 1) * tokens)
        ref, size, plain, _ = _attend_ref(q[one], k[f * states:(f + 1) * states], v[f * states:(f + 1) * states], 1,
                                          q_rows=tokens, k_rows=states)
        tol = (2 * _u(BF16) + 2.0**-15) * size + 2.0**-25 * (plain + 1)
        assert ((out[one].double() - ref).abs() <= tol).all()
    st.close()
