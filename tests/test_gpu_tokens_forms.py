"""Every form in which the token operators are carried out, against plain implementations in 64 bits: which one a call
takes follows from its sizes, and each case here asserts the one that it is meant for (octo_rotate_plan, octo_attend_plan),
so that a change of those rules cannot leave a kernel untested.  Tolerances as in test_gpu_tokens."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2502_01277_b200 as octo
from paper_2502_01277_b200 import binding as B
from test_gpu_tokens import (BF16, F16, F32, _attend_check, _attend_ref, _gen, _ints, _qkv, _rotate_check, _rotate_ref, _u)

pytestmark = pytest.mark.gpu


class _Forms:
    """The library, with a note of how each call was carried out."""

    def __init__(self, lib):
        self._lib, self.seen = lib, []

    def __getattr__(self, name):
        return getattr(self._lib, name)

    def octo_cross_attention(self, args, *rest):
        tile, splits = ctypes.c_int32(-1), ctypes.c_int32(-1)
        assert self._lib.octo_attend_plan(args, ctypes.byref(tile), ctypes.byref(splits)) == B.OCTO_OK
        self.seen.append((tile.value, splits.value))
        return self._lib.octo_cross_attention(args, *rest)

    def octo_norm_rotate(self, args, *rest):
        run, per, flight = (ctypes.c_int32(-1) for _ in range(3))
        assert self._lib.octo_rotate_plan(args, ctypes.byref(run), ctypes.byref(per), ctypes.byref(flight)) == B.OCTO_OK
        self.seen.append((run.value, per.value, flight.value))
        return self._lib.octo_norm_rotate(args, *rest)


@pytest.fixture
def forms(monkeypatch):
    f = _Forms(B.load_library())
    monkeypatch.setattr(B, "load_library", lambda *a: f)
    return f


# ---- attention: tiles ----------------------------------------------------------------------------------------------

def _tile_check(forms, q, k, v, n, **kw):
    out = _attend_check(q, k, v, n, **kw)
    assert forms.seen[-1][0] == 1, "not the kernel for many rows"
    return out


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim,n,q_rows", [(64, 1, 3000), (128, 1, 1700), (64, 6, 700), (72, 2, 1000)])
@pytest.mark.parametrize("masked", [False, True])
def test_tiles_row_maxima(forms, dtype, dim, n, q_rows, masked):
    """Scores that grow along the keys by far more than the weights' room (2^10 a turn), fall, jump once, are equal; a
    negative and a zero scale: the running reference moves, and with it the sums in tensor memory."""
    k_rows = 1500
    q, k, v = _qkv(5, n * q_rows, n * k_rows, 2, 2, dim, dtype)
    mask = None
    if masked:
        mask = (torch.rand(n * k_rows, generator=_gen(2), device="cuda") < 0.5).to(torch.uint8)
        mask[:k_rows // 2 + 13] = 1  # a run, then single keys
    kw = dict(q_rows=q_rows, k_rows=k_rows, key_mask=mask)
    grow = torch.linspace(-3, 3, k_rows, device="cuda").repeat(n)[:, None, None]
    kk, qq = (k.float().abs() * grow).to(dtype), q.abs()
    for scale in (None, -dim ** -0.5, 0.0):
        _tile_check(forms, qq, kk, v, n, scale=scale, **kw)
    _tile_check(forms, qq, kk.flip(0), v, n, **kw)
    jump = k.clone()
    jump.view(n, k_rows, 2, dim)[:, 900] = (3 * k.view(n, k_rows, 2, dim)[:, 900].abs().float()).to(dtype)
    _tile_check(forms, qq, jump, v, n, **kw)
    _tile_check(forms, q, k[:1].expand(n * k_rows, -1, -1), v, n, **kw)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv,dim", [(1, 1, 8), (2, 2, 64), (4, 1, 128), (6, 2, 80), (3, 3, 40), (8, 8, 72), (32, 8, 128)])
@pytest.mark.parametrize("q_rows,k_rows", [(17, 1), (17, 128), (49, 15), (49, 64), (130, 65), (130, 257), (257, 129), (300, 450)])
def test_tiles_uniform(forms, dtype, heads, kv, dim, q_rows, k_rows):
    """Rows and keys around the sizes of halves, tiles and turns; as many segments as make the call one for tiles."""
    n = 3
    while True:
        q, k, v = _qkv(q_rows + k_rows, n * q_rows, n * k_rows, heads, kv, dim, dtype, fused=dim % 16 == 0)
        octo.cross_attention(q, k, v, n, q_rows=q_rows, k_rows=k_rows)
        if forms.seen[-1][0]:
            break
        n = n * 3 // 2
    out = _tile_check(forms, q, k, v, n, q_rows=q_rows, k_rows=k_rows)
    mask = (torch.rand(n * k_rows, generator=_gen(n), device="cuda") < 0.7).to(torch.uint8)
    mask[:k_rows] = 0
    _tile_check(forms, q, k, v, n, q_rows=q_rows, k_rows=k_rows, key_mask=mask)
    assert torch.equal(out, octo.cross_attention(q, k, v, n, q_rows=q_rows, k_rows=k_rows))


@pytest.mark.parametrize("dim", [64, 128])
def test_tiles_visible_nan_and_infinities_come_through(forms, dim):
    q_rows = 6000
    q, k, v = _qkv(6, q_rows, 600, 1, 1, dim, BF16)
    kw = dict(q_rows=q_rows, k_rows=600)
    v[137, 0, 3], v[599, 0, 7] = math.nan, -math.inf
    out = octo.cross_attention(q, k, v, 1, **kw)
    assert torch.isnan(out[:, 0, 3]).all() and (out[:, 0, 7] == -math.inf).all()
    others = [i for i in range(dim) if i not in (3, 7)]
    assert torch.isfinite(out[:, 0, others]).all()
    _, _, clean = _qkv(6, q_rows, 600, 1, 1, dim, BF16)
    for key in (0, 70, 599):
        k2 = k.clone()
        k2[key] = math.nan
        assert torch.isnan(octo.cross_attention(q, k2, clean, 1, **kw)).all()
    assert all(tile == 1 for tile, _ in forms.seen)


@pytest.mark.parametrize("q_rows", [20000])
def test_tiles_without_any_key(forms, q_rows):
    q, k, v = _qkv(0, 2 * q_rows, 0, 4, 2, 64, BF16)
    assert (octo.cross_attention(q, k, v, 2, q_rows=q_rows) == 0).all()
    q, k, v = _qkv(0, 2 * q_rows, 600, 4, 2, 64, BF16)
    k.fill_(math.nan), v.fill_(math.nan)
    out = octo.cross_attention(q, k, v, 2, q_rows=q_rows, k_rows=300, key_mask=torch.zeros(600, dtype=torch.bool, device="cuda"))
    assert (out == 0).all() and all(tile == 1 for tile, _ in forms.seen)


@pytest.mark.parametrize("dim", [64, 128])
def test_tiles_windows_and_bounds(forms, dim):
    """A window of the item list (first), and segments longer than the bounds that the caller gives."""
    q_rows = 1500
    qo, ko = [0, 4, 9, 9, 15], [5, 10, 30, 31, 60]
    q, k, v = _qkv(1, 8 * q_rows, 40 * 8, 4, 2, dim, BF16)
    kw = dict(q_offsets=_ints(qo), k_offsets=_ints(ko), q_rows=q_rows, k_rows=8)
    _tile_check(forms, q, k, v, 4, q_first=3, k_first=7, **kw)
    _tile_check(forms, q, k, v, 4, q_first=-1, k_first=20, max_q=2 * q_rows, max_k=33, **kw)
    _tile_check(forms, q, k, v, 3, q_rows=2 * q_rows, k_rows=120, q_first=1, k_first=-1)


def test_tiles_64_bit_offsets(forms):
    """Keys that lie more than 2^32 elements behind the first."""
    k_total, kv, dim = 1100, 1, 64
    apart = (1 << 32) // 1024
    store = torch.zeros((1 << 32) + 80 * apart, dtype=BF16, device="cuda")
    k = torch.as_strided(store, (k_total, kv, dim), (apart, dim, 1), 0)
    v = torch.as_strided(store, (k_total, kv, dim), (apart, dim, 1), 1024)
    g = _gen(9)
    k.copy_(torch.randn((k_total, kv, dim), generator=g, device="cuda"))
    v.copy_(torch.randn((k_total, kv, dim), generator=g, device="cuda"))
    q = torch.randn((2500, 2, dim), generator=g, device="cuda").to(BF16)
    mask = torch.ones(k_total, dtype=torch.uint8, device="cuda")
    mask[5:900:3] = 0
    for m in (None, mask):
        _tile_check(forms, q, k, v, 1, q_rows=2500, k_rows=k_total, key_mask=m)
    del store, k, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,q_rows,k_rows,heads,kv", [(1, 100, 30000, 2, 1), (1, 700, 8192, 1, 1), (3, 130, 9001, 4, 2)])
def test_tiles_split_over_the_keys(forms, dtype, n, q_rows, k_rows, heads, kv):
    q, k, v = _qkv(n, n * q_rows, n * k_rows, heads, kv, 128, dtype)
    _tile_check(forms, q, k, v, n, q_rows=q_rows, k_rows=k_rows)
    mask = torch.ones(n * k_rows, dtype=torch.uint8, device="cuda")
    mask[100:5000] = 0
    mask[6000:7000:2] = 0
    _tile_check(forms, q, k, v, n, q_rows=q_rows, k_rows=k_rows, key_mask=mask)
    rising = torch.linspace(-2, 2, k_rows, device="cuda").repeat(n)[:, None, None]
    _tile_check(forms, q.abs(), (k.float().abs() * rising).to(dtype), v, n, q_rows=q_rows, k_rows=k_rows)
    assert all(splits > 1 for _, splits in forms.seen)


def test_steps_split_and_whole(forms):
    """The kernel for few rows, with one and with more rows than eight, whole and split."""
    for q_rows, k_rows, heads, kv in [(1, 60, 8, 8), (1, 9001, 8, 1), (3, 9001, 12, 3), (2, 300, 16, 2)]:
        q, k, v = _qkv(k_rows, 2 * q_rows, 2 * k_rows, heads, kv, 64, BF16)
        _attend_check(q, k, v, 2, q_rows=q_rows, k_rows=k_rows)
        assert forms.seen[-1][0] == 0 and (forms.seen[-1][1] > 1) == (k_rows > 1000)


def test_crops_of_a_stage_in_tiles(forms):
    """Tokens of a window of a branch's items, as many as make tiles, to the states of their own frames."""
    import workloads
    from gpu_harness import make_stage, upload_frames
    b = workloads.make_batch("two_branch", batch=3)
    st = make_stage(b.workload, b.n, branches=((224, 224), (64, 32)))
    frames, head = upload_frames(b.frames), torch.from_numpy(b.head).cuda()
    st.preprocess(frames, b.sizes)
    st.postprocess(head)
    cap, first, tokens, states = 400, 3, 49, 700
    _, offsets, n_items = st.crop(0, cap, first_item=first)
    packed = int(n_items[0])
    assert packed > 8
    g = _gen(first)
    q = torch.randn((cap * tokens, 4, 64), generator=g, device="cuda").to(BF16)
    k, v = (torch.randn((b.n * states, 2, 64), generator=g, device="cuda").to(BF16) for _ in range(2))
    _tile_check(forms, q, k, v, b.n, q_offsets=offsets, q_rows=tokens, k_rows=states, q_first=first)
    st.close()


# ---- norm and rotation: heads in flight -----------------------------------------------------------------------------

def _rotate_case(rows, heads, kv, dim, pairs, dtype, seed):
    g = _gen(seed)
    qkv = torch.randn((rows, heads + kv, dim), generator=g, device="cuda").to(dtype)
    pos = torch.rand((rows, 3), generator=g, device="cuda") * torch.tensor([16777216.0, 1080.0, 1.0], device="cuda")
    freqs = torch.rand(pairs, generator=g, device="cuda") * 2
    axes = torch.randint(0, 3, (pairs,), generator=g, device="cuda").int()
    if pairs > 8:
        axes[1], axes[3] = -1, 3  # no axis of these numbers: the pairs stay
    w = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(dtype)
    x = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(dtype)
    return qkv, pos, freqs, axes, w, x


# (heads, kv, dim, pairs): all heads of a token in one warp, in flight one, two or four; the last group of heads not full
# in some; queries and keys of one warp under weights of their own
MANY = [(F16, 16, 16, 64, 32, 8, 4), (BF16, 7, 3, 64, 32, 8, 4), (F16, 6, 1, 128, 32, 8, 4), (F16, 5, 5, 64, 32, 8, 2),
        (BF16, 4, 3, 96, 24, 8, 2), (F16, 1, 1, 64, 32, 8, 1), (F16, 7, 3, 72, 36, 4, 2), (BF16, 3, 2, 254, 127, 1, 2),
        (F16, 1, 1, 254, 100, 1, 1), (F32, 16, 16, 64, 32, 8, 2), (F32, 7, 3, 72, 24, 4, 2), (F32, 1, 1, 72, 18, 2, 1),
        (F32, 5, 5, 64, 16, 8, 2), (BF16, 9, 2, 20, 10, 2, 2), (F16, 6, 3, 36, 9, 1, 2)]


@pytest.mark.parametrize("dtype,heads,kv,dim,pairs,run,flight", MANY)
@pytest.mark.parametrize("ilv", [False, True])
@pytest.mark.parametrize("weights", ["q", "k", "both", "none"])
def test_rotation_of_many_tokens(forms, dtype, heads, kv, dim, pairs, run, flight, ilv, weights):
    rows = 20011
    qkv, pos, freqs, axes, w, x = _rotate_case(rows, heads, kv, dim, pairs, dtype, dim + heads)
    q, k = qkv[:, :heads], qkv[:, heads:]
    wq, wk = (w if weights in ("q", "both") else None), (x if weights in ("k", "both") else None)
    qo, ko = octo.norm_rotate(q, k, pos, freqs, axes, q_weight=wq, k_weight=wk, eps=1e-5, interleaved=ilv)
    got_run, per, got_flight = forms.seen[-1]
    assert per == heads + kv and got_flight == flight and (ilv or got_run == run)
    for got, a, b in ((qo, q, wq), (ko, k, wk)):
        want, size = _rotate_ref(a, b, pos, freqs, axes, 1e-5, ilv)
        _rotate_check(got, want, size, dtype)
    if weights == "both":  # in place, and rows that no item fills
        n = _ints([2001])
        before = qkv.clone()
        octo.norm_rotate(q, k, pos, freqs, axes, q_weight=wq, k_weight=wk, eps=1e-5, interleaved=ilv, n_items=n, item_rows=7,
                         out=(q, k))
        assert torch.equal(q[:14007], qo[:14007]) and torch.equal(k[:14007], ko[:14007])
        assert torch.equal(qkv[14007:], before[14007:])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("heads,kv,dim,pairs", [(16, 16, 64, 32), (13, 6, 64, 32), (7, 5, 72, 24), (9, 0, 128, 64), (11, 4, 254, 127)])
@pytest.mark.parametrize("ilv", [False, True])
def test_rotation_with_the_heads_of_a_token_on_several_warps(forms, dtype, heads, kv, dim, pairs, ilv):
    """More than one head a warp and fewer than all: groups that lie over the border of queries and keys, and a last group
    that is not full."""
    seen = set()
    for rows in (300, 700, 1500, 4000, 9000, 15000):
        qkv, pos, freqs, axes, w, x = _rotate_case(rows, heads, kv, dim, pairs, dtype, rows)
        q, k = qkv[:, :heads], qkv[:, heads:] if kv else None
        qo, ko = octo.norm_rotate(q, k, pos, freqs, axes, q_weight=w, k_weight=x if kv else None, eps=1e-5, interleaved=ilv)
        if not 1 < forms.seen[-1][1] < heads + kv:
            continue
        seen.add(forms.seen[-1][1])
        for got, a, b in ((qo, q, w), (ko, k, x)):
            if a is not None:
                want, size = _rotate_ref(a, b, pos, freqs, axes, 1e-5, ilv)
                _rotate_check(got, want, size, dtype)
    assert seen, "no call had several heads on a warp and not all"


# ---- positions: a warp or a CTA per item ----------------------------------------------------------------------------

def _fits(rec, slot, keep):
    """Size and place of the images, in whole numbers."""
    ow, oh = slot
    cw, ch = (rec[:, 4] - rec[:, 2]).astype(object), (rec[:, 5] - rec[:, 3]).astype(object)
    out = []
    for w, h in zip(cw, ch):
        nw, nh = ow, oh
        if keep and w > 0 and h > 0:
            if ow * h <= oh * w:
                nh = max(1, (2 * ow * h + w) // (2 * w))
            else:
                nw = max(1, (2 * oh * w + h) // (2 * h))
        out.append((nw, nh, (ow - nw) // 2, (oh - nh) // 2))
    return np.array(out, dtype=np.int64)


def _places(rec, slot, p, keep, times):
    """Positions in 64 bits and visibility of all items' patches."""
    rec = rec.astype(np.int64)
    gw, gh = slot[0] // p, slot[1] // p
    fit = _fits(rec, slot, keep)
    good = (rec[:, 4] > rec[:, 2]) & (rec[:, 5] > rec[:, 3]) & (rec[:, 0] >= 0)
    if times is not None:
        good &= rec[:, 0] < len(times)

    def along(count, origin, size, n, pad):
        g = np.arange(count)[None]
        at = origin[:, None] + ((2 * g + 1) * p - 2 * pad[:, None]) * size[:, None] / (2 * n[:, None])
        return at, (g * p < pad[:, None] + n[:, None]) & ((g + 1) * p > pad[:, None])

    x, vx = along(gw, rec[:, 2], rec[:, 4] - rec[:, 2], fit[:, 0], fit[:, 2])
    y, vy = along(gh, rec[:, 3], rec[:, 5] - rec[:, 3], fit[:, 1], fit[:, 3])
    pos = np.zeros((len(rec), gh, gw, 3))
    if times is not None:
        pos[..., 0] = np.where(good, times[np.clip(rec[:, 0], 0, len(times) - 1)], 0)[:, None, None]
    pos[..., 1], pos[..., 2] = y[:, :, None], x[:, None, :]
    pos[~good] = 0
    vis = (vy[:, :, None] & vx[:, None, :] & good[:, None, None]).astype(np.uint8)
    return pos.reshape(len(rec), gh * gw, 3), vis.reshape(len(rec), gh * gw)


@pytest.mark.parametrize("slot,patch", [((224, 224), 16), ((96, 33), 3), ((2048, 16), 8), ((64, 2048), 64), ((24, 40), 8),
                                        ((8, 1), 1), ((2048, 8), 1)])
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("n", [37, 301, 1000])
def test_positions_of_batches(slot, patch, keep, n):
    """Batches that give a warp to an item (from two items per SM on, unless an item's table is long), with times, records that
    are no items between good ones, a count that ends inside a CTA, outputs at odd places, and rectangles up to 2^30 a side."""
    rng = np.random.default_rng(n + patch)
    rec = np.zeros((n, 8), np.int32)
    rec[:, 0] = rng.integers(0, 5, n)
    rec[:, 2:4] = rng.integers(0, 9000, (n, 2))
    rec[:, 4:6] = rec[:, 2:4] + np.exp(rng.uniform(0, math.log(16384), (n, 2))).astype(np.int32)
    far = rng.choice(n, n // 4, replace=False)
    rec[far, 4:6] = rec[far, 2:4] + np.exp(rng.uniform(math.log(1 << 17), math.log(1 << 30), (len(far), 2))).astype(np.int32)
    for k, at in enumerate(rng.choice(n, 12, replace=False)):
        if k % 3 == 0:
            rec[at, 4] = rec[at, 2] - k  # an empty rectangle
        else:
            rec[at, 0] = (-1, 5)[k % 2]  # no frame of that number
    items, packed = torch.from_numpy(rec).cuda(), n - 3
    patches = (slot[0] // patch) * (slot[1] // patch)
    times = (rng.random(5) * 1e5).astype(np.float32)
    want, wvis = _places(rec, slot, patch, keep, times)
    for off in (0, 1):
        pos = torch.full((n * patches * 3 + 4,), -5.0, device="cuda")[off:off + n * patches * 3]
        vis = torch.full((n * patches + 4,), 9, dtype=torch.uint8, device="cuda")[off:off + n * patches]
        octo.patch_positions(items, slot, patch, keep_aspect=keep, times=torch.from_numpy(times).cuda(), n_items=_ints([packed]),
                             positions=pos, visible=vis)
        assert (pos[packed * patches * 3:] == -5).all() and (vis[packed * patches:] == 9).all()
        assert np.array_equal(vis[:packed * patches].cpu().numpy(), wvis[:packed].reshape(-1))
        got = pos[:packed * patches * 3].cpu().numpy().astype(np.float64)
        ref = want[:packed].reshape(-1)
        assert (np.abs(got - ref) <= 2.0**-24 * np.abs(ref) * (1 + 1e-6) + 1e-9).all()
