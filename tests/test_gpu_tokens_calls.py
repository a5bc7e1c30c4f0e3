"""Calls of the token operators that their documentation allows and that went wrong, or were held right by time alone, once.
Tolerances as in test_gpu_tokens."""
import math

import pytest
import torch

import paper_2502_01277_b200 as octo
from test_gpu_tokens import BF16, F16, F32, _attend_ref, _gen, _ints, _qkv, _rotate_check, _rotate_ref, _u

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


@pytest.mark.parametrize("which", ["attention", "rotation", "positions", "stage"])
def test_inputs_of_a_call_on_another_stream_may_be_let_go_of(which):
    """What a call on a given stream reads stays what it is until that stream has read it, although the caller drops
    it and the current stream hands its memory out again."""
    g = _gen(21)
    q, k, v = _qkv(21, 40, 900, 4, 2, 64, BF16)
    pos = torch.rand((40, 1), generator=g, device="cuda") * 100
    freqs, axes = torch.rand(32, generator=g, device="cuda"), torch.zeros(32, dtype=torch.int32, device="cuda")
    mask = (torch.rand(900, generator=g, device="cuda") < 0.5).to(torch.uint8)
    weight = torch.rand(64, generator=g, device="cuda").to(BF16)
    items = torch.zeros((64, 8), dtype=torch.int32, device="cuda")
    items[:, 4:6] = 100
    times = torch.rand(1, generator=g, device="cuda")
    st = None
    if which == "attention":
        given = [q, k, v, _ints([0, 3, 10]), _ints([0, 400, 900]), mask]
        call = lambda s, q, k, v, qo, ko, m: (octo.cross_attention(q, k, v, 2, q_offsets=qo, k_offsets=ko, q_rows=4, key_mask=m,
                                                                   stream=s),)
    elif which == "rotation":
        given = [q, k[:40], pos, freqs, axes, weight, weight + 1, _ints([40])]
        call = lambda s, q, k, p, f, a, w, x, n: octo.norm_rotate(q, k, p, f, a, q_weight=w, k_weight=x, n_items=n, stream=s)
    elif which == "positions":
        given = [items, times, _ints([64])]
        call = lambda s, i, t, n: octo.patch_positions(i, (224, 224), 16, times=t, n_items=n, stream=s)
    else:
        import workloads
        from gpu_harness import make_stage, upload_frames
        b = workloads.make_batch("two_branch", batch=3)
        st = make_stage(b.workload, b.n)
        frames, head = upload_frames(b.frames), torch.from_numpy(b.head).cuda()
        st.preprocess(frames, b.sizes)
        st.postprocess(head)
        _, _, count = st.crop(0, 8)
        assert int(count[0]) == 8
        given = [torch.tensor([3.0, 4.0, 5.0], device="cuda")]
        call = lambda s, t: st.patch_positions(0, 8, 16, times=t, stream=s)
    want = [w.clone() for w in call(None, *given)]
    side = torch.cuda.Stream()
    for n in range(len(given)):
        args = [x.clone() if i == n else x for i, x in enumerate(given)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        got = call(side, *args)
        args[n] = None
        again = [torch.empty_like(given[n]) for _ in range(64)]  # (many small blocks may be free)
        for x in again:
            x.fill_(77 if x.dtype in (torch.int32, torch.uint8) else 1e4)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n
        del again
    if st is not None:
        st.close()


def test_an_output_of_a_call_on_another_stream_may_be_let_go_of():
    """A result that the caller drops is written by the given stream before its memory is anyone else's."""
    q, k, v = _qkv(22, 64, 900, 4, 2, 64, BF16)
    side = torch.cuda.Stream()
    for use in (lambda o: octo.cross_attention(q, k, v, 1, q_rows=64, k_rows=900, out=o, stream=side),
                lambda o: octo.norm_rotate(q, None, torch.zeros((64, 1), device="cuda"), torch.zeros(32, device="cuda"),
                                           torch.zeros(32, dtype=torch.int32, device="cuda"), out=(o, None), stream=side)):
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        use(out)
        del out
        again = [torch.empty_like(q).fill_(5.0) for _ in range(4)]
        torch.cuda.synchronize()
        assert all((x == 5.0).all() for x in again)
        del again


def test_calls_on_a_forked_stream_inside_a_capture():
    """The same inside a CUDA graph: temporaries of the capturing stream, read on a stream forked from it."""
    q, k, v = _qkv(24, 64, 20000, 4, 2, 64, BF16)
    pos, freqs = torch.rand((64, 1), device="cuda") * 100, torch.rand(32, device="cuda")
    axes = torch.zeros(32, dtype=torch.int32, device="cuda")

    def one_pass(side):
        main = torch.cuda.current_stream()
        turned, _ = octo.norm_rotate(q + q, None, pos, freqs, axes)
        kk, vv = k + k, v + v  # (ready on the other stream: before it waits for this one)
        if side is not None:
            side.wait_stream(main)
        out = octo.cross_attention(turned, kk, vv, 1, q_rows=64, k_rows=20000, stream=side)
        del turned, kk, vv
        if side is not None:
            main.wait_stream(side)
        return out

    want = one_pass(None)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = one_pass(side)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    del graph, out
    assert torch.equal(one_pass(side), want)


@pytest.mark.parametrize("q_rows", [1, 6000])
def test_attention_scale_zero_is_the_mean_whatever_the_scores(q_rows):
    """Scores up to 2^125."""
    q, k, v = _qkv(23, q_rows, 1500, 2, 2, 64, BF16)
    q, k = torch.sign(q) * 2.0**60, torch.sign(k) * 2.0**59
    out = octo.cross_attention(q, k, v, 1, q_rows=q_rows, k_rows=1500, scale=0.0)
    want, size = v.double().mean(0), v.double().abs().mean(0)
    assert ((out.double() - want).abs() <= (2 * _u(BF16) + 2.0**-15) * size).all()


def test_attention_looks_through_a_billion_hidden_keys():
    """One segment of 2^30 - 1196 keys, all hidden, which takes seconds to look through, beside 299 of four keys: waiting that
    long is not a wait that has run out.  (The keys are one row in memory, seen again and again.)"""
    n, q_rows, dim = 300, 32, 8
    first = (1 << 30) - 4 * (n - 1)
    g = _gen(25)
    q = torch.randn((n * q_rows, 1, dim), generator=g, device="cuda").to(BF16)
    k, v = (torch.randn((1, 1, dim), generator=g, device="cuda").to(BF16).expand(1 << 30, 1, dim) for _ in range(2))
    mask = torch.zeros(1 << 30, dtype=torch.uint8, device="cuda")
    mask[first:] = 1
    offsets = _ints([0] + [first + 4 * i for i in range(n)])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = octo.cross_attention(q, k, v, n, q_rows=q_rows, k_offsets=offsets, key_mask=mask, status=status)
    assert int(status) == 0
    assert (out[:q_rows] == 0).all()
    assert ((out[q_rows:].double() - v[:1].double()).abs() <= (2 * _u(BF16) + 2.0**-15) * v[:1].double().abs()).all()
    del mask
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("turns", [0.5, 16.0, 2.0**12, 2.0**22, 2.0**27])
@pytest.mark.parametrize("whole", [False, True])
def test_sine_and_cosine_of_the_rotation(dtype, turns, whole):
    """Cosine and sine, read from heads of (1, 0), against the stated bounds.

    binary32: two units of sincospif (2^-22) and the angle, taken off its whole turns with 2^-46 of them (2 pi 2^-46 turns;
    beyond 2^22 turns in binary64, 2^-51).  16 bits: __sinf and __cosf are off by up to 2^-21.19 (4.2e-7); the turns' rest is
    rounded to binary32 once (2^-25 turns, 1.9e-7; near 2^22 turns 2^-24, 3.8e-7) and multiplied by 2 pi (half a step below 4,
    1.2e-7, and the constant's 2^-25.1 of up to pi, 0.9e-7), and the reduction is off by up to 3.8e-7 there: 1.4e-6 in all.  The
    output's rounding hides that except near the zeros, which is where a part of these angles lies."""
    rows, pairs = 60000, 128
    g = _gen(int(turns) + 7)
    q = torch.zeros((rows, 1, 2 * pairs), device="cuda", dtype=dtype)
    q[..., :pairs] = 1
    pos = torch.randint(-(1 << 24), 1 << 24, (rows, 1), generator=g, device="cuda").int()
    freqs = torch.rand(pairs, generator=g, device="cuda") * (turns * 2 * math.pi / 2**24)
    axes = torch.zeros(pairs, dtype=torch.int32, device="cuda")
    out, _ = octo.norm_rotate(q, None, pos if whole else pos.float(), freqs, axes)
    angle = pos.double() * freqs.double()  # (exact)
    want = torch.cat([angle.cos(), angle.sin()], -1)
    off = 2 * math.pi * min(turns * 2.0**-46, 2.0**-24) + turns * 2 * math.pi * 2.0**-51
    tol = 2.0**-22 + off if dtype == F32 else 1.4e-6 + turns * 2 * math.pi * 2.0**-51
    tol = tol + _u(dtype) * want.abs() + (2.0**-25 if dtype == F16 else 0.0)
    err = (out[:, 0].double() - want).abs()
    assert (err <= tol).all(), float((err - tol).max())
    assert int((want.abs() < 2.0**-12).sum()) > 1000


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rotation_by_the_ends_of_int32(dtype):
    """(The smallest int32 has no absolute value.)"""
    ends = [-(1 << 31), -(1 << 31) + 1, (1 << 31) - 1, -(1 << 24) - 1, -(1 << 24), (1 << 24) + 1, 0]
    pos, g = _ints([[p] for p in ends]), _gen(31)
    q = torch.randn((len(ends), 2, 64), generator=g, device="cuda").to(dtype)
    freqs, axes = torch.rand(32, generator=g, device="cuda") * 2.0**-20, torch.zeros(32, dtype=torch.int32, device="cuda")
    out, _ = octo.norm_rotate(q, None, pos, freqs, axes)
    want, size = _rotate_ref(q, None, pos, freqs, axes, 1e-6, False)
    _rotate_check(out, want, size, dtype)


def test_refusals_are_the_frameworks_own():
    """Sizes of none and negative counts are refused as every other argument is, not by what trips over them."""
    import workloads
    from gpu_harness import make_stage, upload_frames
    b = workloads.make_batch("two_branch", batch=3)
    st = make_stage(b.workload, b.n)
    frames, head = upload_frames(b.frames), torch.from_numpy(b.head).cuda()
    st.preprocess(frames, b.sizes)
    st.postprocess(head)
    st.crop(0, 8)
    q, k, v = _qkv(0, 4, 8, 4, 2, 64, BF16)
    for call in (lambda: st.patch_positions(0, -1, 16), lambda: st.patch_positions(-1, 8, 16),
                 lambda: octo.cross_attention(q[..., :0], k[..., :0], v[..., :0], 1, k_rows=8),
                 lambda: octo.cross_attention(q, k, v, 1, k_rows=8, out=q[:1].expand(4, -1, -1)),
                 lambda: octo.norm_rotate(q, None, torch.zeros((4, 1), device="cuda"), torch.zeros(2, device="cuda"),
                                          _ints([0, 0]), out=(q[:1].expand(4, -1, -1), None))):
        with pytest.raises(octo.OctoError) as e:
            call()
        assert e.value.code == octo.binding.OCTO_E_INVALID_ARG
    st.close()
