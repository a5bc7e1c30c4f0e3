"""What a transformer behind a cascade stage has the library do, as cases that can be timed.

Three operators, each measured alone: where the patches of packed crops lie in time and in their
source frames (patch_positions), the norm of queries and keys per head together with their rotation by
those positions (norm_rotate), and the attention of one set of tokens to another set's states, segment by
segment (cross_attention).  The number of items of a frame is known on the device only, so the operators
take the stage's item table, offsets and counts as they lie there.  Crop sizes, frame sizes and numbers of
detections are those of the repository's workloads; head layouts are generic."""
from __future__ import annotations

import json
import math
import random

import torch

own = False

_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
_EPS = 1e-6

# positions: `slots` places for crops, `items` of them packed; slot size and patch side in pixels
_POSITIONS = dict(kind="positions", frames=1, slots=32, items=22, slot_w=224, slot_h=224, patch=16, fit=False)
# rotate: `slots` items of `rows` tokens each, `items` of them packed; `rotated` leading elements of a head turn
_ROTATE = dict(kind="rotate", slots=22, items=22, rows=1, heads=16, kv_heads=16, dim=64, rotated=64, axes=3, dtype="fp16",
               norm=True, interleaved=False, fused=True)
# attend: n segments.  objects > 0: about that many items of q_rows tokens in a segment (offsets on the device, slots
# beyond the last item); 0: q_rows query rows in every segment.  Keys: k_rows in every segment, or up to k_rows (ragged).
# hidden: share of the keys that the mask takes away.
_ATTEND = dict(kind="attend", n=1, objects=0, q_rows=1, k_rows=196, ragged=False, hidden=0.0, heads=16, kv_heads=16, dim=64,
               dtype="fp16", fused=True)


def _positions(**kw):
    return {**_POSITIONS, **kw}


def _rotate(**kw):
    return {**_ROTATE, **kw}


def _attend(**kw):
    return {**_ATTEND, **kw}


def listed():
    return [
        # the crops of one camera frame: a handful of items, where the launch is all there is
        _positions(name="positions_camera"),
        # a throughput server's batch of fitted crops
        _positions(name="positions_server", frames=256, slots=8192, items=7356, fit=True),
        # one new token for each object of a camera frame (a plate being read out)
        _rotate(name="rotate_step", slots=22, items=22, rows=1),
        # the 40 x 40 patches of one 640 x 640 detector canvas, queries grouped over fewer keys
        _rotate(name="rotate_frame", slots=1, items=1, rows=1600, heads=32, kv_heads=8, dim=128, rotated=128, dtype="bf16"),
        # the 14 x 14 patches of the crops of 64 frames
        _rotate(name="rotate_crops", slots=1408, items=1401, rows=196),
        # odd sizes: heads of 72 of which 48 elements turn in pairs side by side, two axes, binary32, no norm
        _rotate(name="rotate_odd", slots=149, items=149, rows=67, heads=12, kv_heads=2, dim=72, rotated=48, axes=2, dtype="fp32",
                norm=False, interleaved=True, fused=False),
        # one new token for each of a camera frame's objects against the states of its crop
        _attend(name="attend_step", n=22, q_rows=1, k_rows=196, heads=8, kv_heads=8),
        # one new token for each of 64 cameras against the states of its frame
        _attend(name="attend_step_frames", n=64, q_rows=1, k_rows=1600, heads=32, kv_heads=8, dim=128, dtype="bf16"),
        # questions of a few tokens about clips of different length; patches that show only canvas are hidden
        _attend(name="attend_clips", n=5, q_rows=3, k_rows=59200, ragged=True, hidden=0.4375, heads=32, kv_heads=8, dim=128,
                dtype="bf16"),
        # the 7 x 7 tokens of every crop attend to the states of the frame it was cut from, canvas hidden
        _attend(name="attend_crops", n=64, objects=22, q_rows=49, k_rows=1600, hidden=0.4375),
        # the 14 x 14 tokens of every crop attend to the states of its frame, wide heads
        _attend(name="attend_crops_wide", n=32, objects=22, q_rows=196, k_rows=1600, dim=128, dtype="bf16"),
        # odd sizes: heads of 80, three queries a key head, states of uneven length
        _attend(name="attend_odd", n=13, objects=9, q_rows=37, k_rows=777, ragged=True, heads=6, kv_heads=2, dim=80,
                dtype="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["positions", "rotate", "rotate", "attend", "attend", "attend"])
    if kind == "positions":
        patch = rng.choice([8, 14, 16, 28, 32])
        slot_w = patch * rng.choice([k for k in range(1, 41) if patch * k % 8 == 0])
        slot_h = patch * rng.randint(1, 40)
        slots = min(log_int(1, 8192), 8192 * 196 // ((slot_w // patch) * (slot_h // patch)) + 1)
        return _positions(frames=log_int(1, 512), slots=slots, items=rng.randint(1, slots), slot_w=slot_w, slot_h=slot_h,
                          patch=patch, fit=rng.random() < 0.5)
    if kind == "rotate":
        dtype = rng.choice(["fp16", "bf16", "fp32"])
        dim = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 20, 36, 192, 256])
        rotated = rng.choice([dim, dim, dim, dim // 2 // 2 * 2])
        kv = rng.choice([1, 2, 3, 4, 8, 16])
        heads = kv * rng.choice([1, 1, 2, 3, 4])
        rows = rng.choice([1, 1, 49, 196, 256, log_int(1, 4096)])
        most = 500_000_000 // (heads + kv) // dim // rows // (2 if dtype == "fp32" else 1)
        slots = log_int(1, max(2, most))
        return _rotate(slots=slots, items=max(1, slots - rng.choice([0, 0, 1, 7])), rows=rows, heads=heads, kv_heads=kv, dim=dim,
                       rotated=rotated, axes=rng.choice([1, 2, 3]), dtype=dtype, norm=rng.random() < 0.7,
                       interleaved=rng.random() < 0.4, fused=rng.random() < 0.6)
    c = _attend(dim=rng.choice([32, 64, 64, 72, 80, 96, 128, 128]), dtype=rng.choice(["fp16", "bf16"]),
                kv_heads=rng.choice([1, 2, 3, 4, 8, 16]), hidden=rng.choice([0.0, 0.0, 0.25, 0.4375]),
                ragged=rng.random() < 0.5, fused=rng.random() < 0.7)
    c["heads"] = c["kv_heads"] * rng.choice([1, 1, 2, 3, 4, 8])
    if rng.random() < 0.5:  # few queries
        c["n"], c["q_rows"] = log_int(1, 256), rng.choice([1, 1, 1, 2, 4, 7])
        most = 400_000_000 // (c["n"] * c["kv_heads"] * 2 * c["dim"])
    else:
        c["n"], c["objects"], c["q_rows"] = log_int(1, 64), rng.choice([0, 0, 1, 5, 22]), log_int(8, 400)
        if not c["objects"]:
            c["q_rows"] = log_int(16, 4096)
        rows = c["n"] * max(1, c["objects"]) * c["q_rows"]
        most = min(2e12 / (4 * rows * c["heads"] * c["dim"]), 400_000_000 // (c["n"] * c["kv_heads"] * 2 * c["dim"]))
    c["k_rows"] = log_int(1, max(2, min(65536, int(most))))
    return c


# ---- what a case's segments look like: from the case alone, so that every seed has the same work -------------------

def _rng_of(case):
    return random.Random(json.dumps({k: v for k, v in case.items() if k != "name"}, sort_keys=True))


def _lengths(case):
    """Per segment (query rows, key rows), and the number of query slots."""
    rng = _rng_of(case)
    out, slots = [], 0
    for s in range(case["n"]):
        items = 1
        if case["objects"]:
            items = max(0 if s else 1, int(round(rng.gauss(case["objects"], 1.5 * math.sqrt(case["objects"])))))
            if s % 9 == 8:
                items = 0  # a frame without a detection
        keys = case["k_rows"]
        if case["ragged"]:
            keys = 0 if s % 7 == 6 else max(1, int(case["k_rows"] * rng.uniform(0.25, 1.0)))
        out.append((items * case["q_rows"], keys))
        slots += items
    if case["objects"]:
        slots += 5  # places of the batch that no item fills
    return out, max(1, slots) * case["q_rows"]


def work(case):
    if case["kind"] == "positions":
        patches = (case["slot_w"] // case["patch"]) * (case["slot_h"] // case["patch"])
        return {"bytes": case["items"] * (32 + patches * 13) + case["frames"] * 4, "flops": case["items"] * patches * 8}
    size = _TYPES[case["dtype"]].itemsize
    if case["kind"] == "rotate":
        rows = case["items"] * case["rows"]
        elements = rows * (case["heads"] + case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * elements * size + rows * case["axes"] * 4, "flops": 8 * elements}
    segments, _ = _lengths(case)
    rows = sum(q for q, k in segments)
    keys = sum(k for q, k in segments if q)
    pairs = sum(q * k for q, k in segments)
    return {"bytes": size * case["dim"] * (2 * rows * case["heads"] + 2 * keys * case["kv_heads"]) + (keys if case["hidden"] else 0),
            "flops": 4 * pairs * case["heads"] * case["dim"]}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def prepare(case, seed):
    g = _generator(seed)
    state = {"case": case}
    if case["kind"] == "positions":
        # rectangles of detections in 1920 x 1080 frames, in frame order, as the stage's item table holds them
        slots, n = case["slots"], case["frames"]
        frame = torch.sort(torch.randint(0, n, (slots,), generator=g, device="cuda"))[0]
        w = torch.randint(8, 400, (slots,), generator=g, device="cuda")
        h = torch.randint(8, 400, (slots,), generator=g, device="cuda")
        x = (torch.rand(slots, generator=g, device="cuda") * (1920 - w)).long()
        y = (torch.rand(slots, generator=g, device="cuda") * (1080 - h)).long()
        det, zero = torch.arange(slots, device="cuda"), torch.zeros_like(x)
        state["items"] = torch.stack([frame, det, x, y, x + w, y + h, zero, zero], 1).int()
        state["n_items"] = torch.tensor([case["items"], case["items"]], device="cuda", dtype=torch.int32)
        state["times"] = torch.arange(n, device="cuda").float() * 4 + 1000 * torch.rand(1, generator=g, device="cuda")
        patches = (case["slot_w"] // case["patch"]) * (case["slot_h"] // case["patch"])
        state["positions"] = torch.zeros((slots, patches, 3), device="cuda")
        state["visible"] = torch.zeros((slots, patches), device="cuda", dtype=torch.uint8)
        return state
    dtype = _TYPES[case["dtype"]]
    heads, kv, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "rotate":
        rows = case["slots"] * case["rows"]
        if case["fused"]:  # one projection's output: queries, keys and values side by side in a row
            qkv = _normal(g, (rows, heads + 2 * kv, dim), dtype)
            state["q"], state["k"] = qkv[:, :heads], qkv[:, heads:heads + kv]
        else:
            state["q"], state["k"] = _normal(g, (rows, heads, dim), dtype), _normal(g, (rows, kv, dim), dtype)
        state["q_weight"] = (1 + 0.2 * _normal(g, (dim,), torch.float32)).to(dtype) if case["norm"] else None
        state["k_weight"] = (1 + 0.2 * _normal(g, (dim,), torch.float32)).to(dtype) if case["norm"] else None
        # time in frames since the stream began, then pixels of the source frame
        span = torch.tensor([100000.0, 1080.0, 1920.0], device="cuda")[3 - case["axes"]:]
        state["positions"] = torch.rand((rows, case["axes"]), generator=g, device="cuda") * span
        pairs = case["rotated"] // 2
        i = torch.arange(pairs, device="cuda")
        per_axis = -(-pairs // case["axes"])
        state["freqs"] = (10000.0 ** (-(i % per_axis).double() / per_axis)).float()
        state["axes"] = (i // per_axis).int()
        state["n_items"] = torch.tensor([case["items"], case["items"]], device="cuda", dtype=torch.int32)
        state["out"] = (torch.zeros((rows, heads, dim), device="cuda", dtype=dtype),
                        torch.zeros((rows, kv, dim), device="cuda", dtype=dtype))
        return state
    segments, q_total = _lengths(case)
    order = torch.randperm(case["n"], generator=g, device="cuda").tolist()
    segments = [segments[s] for s in order]
    state["segments"], q0, k0 = [], 0, 0
    for q, k in segments:
        state["segments"].append((q0, q0 + q, k0, k0 + k))
        q0, k0 = q0 + q, k0 + k
    q_offsets = [b // case["q_rows"] for b, _, _, _ in state["segments"]] + [q0 // case["q_rows"]]
    state["q_offsets"] = torch.tensor(q_offsets, device="cuda", dtype=torch.int32) if case["objects"] else None
    k_offsets = [b for _, _, b, _ in state["segments"]] + [k0]
    state["k_offsets"] = torch.tensor(k_offsets, device="cuda", dtype=torch.int32) if case["ragged"] else None
    state["q"] = 1.5 * _normal(g, (q_total, heads, dim), dtype)
    keys = max(1, k0)
    if case["fused"]:  # one projection's output: keys and values side by side in a row
        both = _normal(g, (keys, 2, kv, dim), dtype)
        state["k"], state["v"] = both[:, 0], both[:, 1]
    else:
        state["k"], state["v"] = _normal(g, (keys, kv, dim), dtype), _normal(g, (keys, kv, dim), dtype)
    state["mask"] = None
    if case["hidden"]:  # canvas above and below a wide frame: bands of rows in every frame's states
        states = min(1600, case["k_rows"])
        place = torch.arange(keys, device="cuda") % states
        edge = int(states * case["hidden"] / 2)
        state["mask"] = ((place >= edge) & (place < states - edge)).to(torch.uint8)
    state["out"] = torch.zeros_like(state["q"])
    return state


# ---- the passes ----------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        import paper_2502_01277_b200 as octo
        if case["kind"] == "positions":
            return octo.patch_positions(state["items"], (case["slot_w"], case["slot_h"]), case["patch"], keep_aspect=case["fit"],
                                        times=state["times"], n_items=state["n_items"], positions=state["positions"],
                                        visible=state["visible"])
        if case["kind"] == "rotate":
            return octo.norm_rotate(state["q"], state["k"], state["positions"], state["freqs"], state["axes"],
                                    q_weight=state["q_weight"], k_weight=state["k_weight"], eps=_EPS,
                                    interleaved=case["interleaved"], n_items=state["n_items"], item_rows=case["rows"],
                                    out=state["out"])
        ragged_q = state["q_offsets"] is not None
        return octo.cross_attention(state["q"], state["k"], state["v"], case["n"], q_offsets=state["q_offsets"],
                                    k_offsets=state["k_offsets"], q_rows=case["q_rows"],
                                    k_rows=1 if case["ragged"] else case["k_rows"],
                                    max_q=None if ragged_q else case["q_rows"], max_k=case["k_rows"],
                                    key_mask=state["mask"], out=state["out"])
    return {"positions": _plain_positions, "rotate": _plain_rotate, "attend": _plain_attend}[case["kind"]](case, state)


def _fit(case, cw, ch):
    """Image size and place inside the slot, in whole numbers (a plain stretch fills the slot)."""
    ow, oh = case["slot_w"], case["slot_h"]
    if not case["fit"]:
        return torch.full_like(cw, ow), torch.full_like(cw, oh), torch.zeros_like(cw), torch.zeros_like(cw)
    wide = ow * ch <= oh * cw
    nw = torch.where(wide, torch.full_like(cw, ow), ((2 * oh * cw + ch) // (2 * ch)).clamp(min=1))
    nh = torch.where(wide, ((2 * ow * ch + cw) // (2 * cw)).clamp(min=1), torch.full_like(cw, oh))
    return nw, nh, (ow - nw) // 2, (oh - nh) // 2


def _plain_positions(case, state):
    n, p = case["items"], case["patch"]
    frame, _, x0, y0, x1, y1, _, _ = state["items"][:n].long().unbind(1)
    nw, nh, left, top = _fit(case, x1 - x0, y1 - y0)
    i = torch.arange(case["slot_w"] // p, device="cuda")[None]
    j = torch.arange(case["slot_h"] // p, device="cuda")[None]
    # in 64 bits: a centre may lie next to where 32 bits round the other way
    x = x0[:, None] + ((2 * i + 1) * p - 2 * left[:, None]) * (x1 - x0)[:, None] / (2 * nw[:, None]).double()
    y = y0[:, None] + ((2 * j + 1) * p - 2 * top[:, None]) * (y1 - y0)[:, None] / (2 * nh[:, None]).double()
    seen_x = (i * p < (left + nw)[:, None]) & ((i + 1) * p > left[:, None])
    seen_y = (j * p < (top + nh)[:, None]) & ((j + 1) * p > top[:, None])
    gw, gh = x.shape[1], y.shape[1]
    out, visible = state["positions"], state["visible"]
    out[:n, :, 0] = state["times"][frame][:, None]
    out[:n, :, 1] = y.float()[:, :, None].expand(-1, -1, gw).reshape(n, gh * gw)
    out[:n, :, 2] = x.float()[:, None, :].expand(-1, gh, -1).reshape(n, gh * gw)
    visible[:n] = (seen_y[:, :, None] & seen_x[:, None, :]).reshape(n, gh * gw)
    return out, visible


def _plain_rotate(case, state):
    rows, pairs = case["items"] * case["rows"], case["rotated"] // 2
    # in 64 bits: the angle of a far position
    angle = state["positions"][:rows].double()[:, state["axes"].long()] * state["freqs"].double()
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    for x, weight, out in ((state["q"], state["q_weight"], state["out"][0]), (state["k"], state["k_weight"], state["out"][1])):
        y = x[:rows].float()
        if weight is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * weight.float()
        if case["interleaved"]:
            a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
            turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
        else:
            a, b = y[..., :pairs], y[..., pairs:2 * pairs]
            turned = torch.cat([a * c - b * s, b * c + a * s], -1)
        out[:rows] = torch.cat([turned, y[..., 2 * pairs:]], -1).to(x.dtype)
    return state["out"]


def _plain_attend(case, state):
    group, scale = case["heads"] // case["kv_heads"], case["dim"] ** -0.5
    out = state["out"]
    for q0, q1, k0, k1 in state["segments"]:
        if q1 == q0:
            continue
        if k1 == k0:
            out[q0:q1] = 0
            continue
        q = state["q"][q0:q1].float().unflatten(1, (case["kv_heads"], group)).permute(1, 2, 0, 3).flatten(1, 2)
        k = state["k"][k0:k1].float().permute(1, 2, 0)
        v = state["v"][k0:k1].float().transpose(0, 1)
        score = torch.matmul(q, k) * scale
        if state["mask"] is not None:
            score = score.masked_fill(state["mask"][k0:k1] == 0, -math.inf)
        top = score.max(-1, keepdim=True)[0].clamp(min=-3e38)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v) / total.clamp(min=1e-38)
        o = o.unflatten(1, (group, q1 - q0)).permute(2, 0, 1, 3).flatten(1, 2)
        out[q0:q1] = o.to(out.dtype)
    return out


# ---- from the definitions, in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "positions":
        # a patch's centre as a fraction of the image inside its slot, times the rectangle's size
        rec = state["items"].double()
        want, seen = state["positions"].double(), state["visible"].clone()
        ow, oh, p = case["slot_w"], case["slot_h"], case["patch"]
        gw, gh = ow // p, oh // p
        keep = torch.arange(case["slots"], device="cuda") < case["items"]
        cw, ch = rec[:, 4] - rec[:, 2], rec[:, 5] - rec[:, 3]
        nw, nh = torch.full_like(cw, ow), torch.full_like(ch, oh)
        if case["fit"]:
            nw = torch.where(ow * ch <= oh * cw, nw, torch.floor(oh * cw / ch + 0.5).clamp(min=1))
            nh = torch.where(ow * ch <= oh * cw, torch.floor(ow * ch / cw + 0.5).clamp(min=1), nh)
        left, top = torch.floor((ow - nw) / 2), torch.floor((oh - nh) / 2)
        for j in range(gh):
            for i in range(gw):
                row = torch.stack([state["times"].double()[rec[:, 0].long()],
                                   rec[:, 3] + ((j + 0.5) * p - top) / nh * ch, rec[:, 2] + ((i + 0.5) * p - left) / nw * cw], 1)
                want[:, j * gw + i] = torch.where(keep[:, None], row, want[:, j * gw + i])
                inside = (j * p < top + nh) & (j * p + p > top) & (i * p < left + nw) & (i * p + p > left)
                seen[:, j * gw + i] = (keep & inside).to(torch.uint8)
        return want, seen
    if case["kind"] == "rotate":
        rows, half = case["items"] * case["rows"], case["rotated"] // 2
        outs = []
        for name, weight in (("q", "q_weight"), ("k", "k_weight")):
            x = state[name].double()
            want = torch.zeros_like(x)
            for b in range(0, rows, 65536):
                e = min(rows, b + 65536)
                z = x[b:e].clone()
                if case["norm"]:
                    z /= torch.sqrt(z.square().sum(-1, keepdim=True) / case["dim"] + _EPS)
                    z *= state[weight].double()
                r = z.clone()
                for i in range(half):
                    m, n = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
                    phi = (state["positions"][b:e, state["axes"][i].item()].double() * state["freqs"][i].double())[:, None]
                    r[..., m] = z[..., m] * torch.cos(phi) - z[..., n] * torch.sin(phi)
                    r[..., n] = z[..., m] * torch.sin(phi) + z[..., n] * torch.cos(phi)
                want[b:e] = r
            outs.append(want)
        return tuple(outs)
    want = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    group = case["heads"] // case["kv_heads"]
    for q0, q1, k0, k1 in state["segments"]:
        if q1 == q0 or k1 == k0:
            continue
        rows = torch.arange(k0, k1, device="cuda")
        if state["mask"] is not None:
            rows = rows[state["mask"][k0:k1] != 0]
        if not rows.numel():
            continue
        for h in range(case["heads"]):
            k, v = state["k"][rows, h // group].double(), state["v"][rows, h // group].double()
            for b in range(q0, q1, 8192):
                q = state["q"][b:min(q1, b + 8192), h].double()
                want[b:min(q1, b + 8192), h] = torch.softmax(q @ k.T / math.sqrt(case["dim"]), -1) @ v
    return want
