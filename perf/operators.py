"""Decode under eviction by accumulated attention, and the decode cache in 4 bits: cases that can be timed and compared.

A case is a dict of plain values.  ``kind`` says what one pass is:

  accum   ``steps`` generated tokens on a cache whose pool keeps the rows that received the most attention so far
          (lte_attn_decode_accum)
  four    ``steps`` generated tokens on a cache held in 4 bits, then its hand-over to an ordinary cache, as before the next turn's
          prompt (lte_attn_decode4 for ``rule`` "learned", lte_attn_decode4_accum for "accum"; lte_cache4_unpack)
  pack    an ordinary cache put into 4 bits, and back (lte_cache4_pack, lte_cache4_unpack)

H counts key/value heads, G query heads per key/value head; the ring holds W rows, the pool R.  ``n`` tokens have been seen, and the pool
holds ``cnt`` entries (``ragged``: a number of its own, up to cnt, in every head).  K is the number of the learned scorer's taps.

``own`` false: the operators in elementary torch operations on the caches' bytes, whose layout lte.h documents.  ``own`` true: the
library's calls on the same bytes.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": (torch.bfloat16, 1, 2), "f32": (torch.float32, 0, 4)}
GROUP = 32                                                           # channels that share a step and a zero in 4 bits
HEADER = 256


def _case(name, kind, dtype, B, H, G, d, W, R, n, cnt, steps=1, rule="accum", decay=1.0, sink=0, K=7, ragged=False):
    c = {"kind": kind, "dtype": dtype, "B": B, "H": H, "G": G, "d": d, "W": W, "R": R, "n": n, "cnt": cnt, "steps": steps, "rule": rule,
         "decay": decay, "sink": sink, "K": K, "ragged": ragged}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call there is: the heads, window and budget of configuration C1, fp32 (a unit test, a tiny model)
        _case("tiny fp32", "accum", "f32", 1, 2, 1, 32, 16, 8, 60, 8),
        # one user's answer at d = 128, the heads, window and budget of configuration C3: latency counts
        _case("one answer d128", "accum", "bf16", 1, 16, 1, 128, 512, 512, 3000, 512, steps=4),
        # batched decode, configuration C4
        _case("batch C4", "accum", "bf16", 128, 16, 1, 64, 128, 128, 2048, 128),
        # the paper's serving shape: 32 query heads on 8, window 768, budget 512, sink tokens; the pools fill at their own pace and
        # old attention fades
        _case("serving", "accum", "bf16", 32, 8, 4, 64, 768, 512, 2000, 512, sink=4, decay=0.98, ragged=True),
        # one long document: a pool of 16,384 rows
        _case("long pool", "accum", "bf16", 1, 8, 4, 128, 1024, 16384, 40000, 16384),
        # odd sizes, a last query that alone decides
        _case("odd sizes", "accum", "bf16", 3, 5, 3, 128, 301, 77, 1000, 77, decay=0.0, sink=1),
        # the smallest call in 4 bits, the ring not yet full
        _case("tiny fp32 in 4 bits", "four", "f32", 1, 2, 1, 32, 16, 8, 11, 0, steps=2, rule="learned", K=5),
        # one user's answer in 4 bits, learned eviction
        _case("one answer d128 in 4 bits", "four", "bf16", 1, 16, 1, 128, 512, 512, 3000, 512, steps=8, rule="learned"),
        # batched decode in 4 bits, learned eviction
        _case("batch C4 in 4 bits", "four", "bf16", 128, 16, 1, 64, 128, 128, 2048, 128, steps=16, rule="learned"),
        # the serving shape in 4 bits, accumulated attention
        _case("serving in 4 bits", "four", "bf16", 32, 8, 4, 64, 768, 512, 5000, 512, steps=16, sink=4),
        # caches of the serving shape and of a small odd one, on their way into 4 bits and back
        _case("pack serving", "pack", "bf16", 32, 8, 4, 64, 768, 512, 5000, 512, sink=4),
        _case("pack odd fp32", "pack", "f32", 3, 5, 1, 128, 77, 41, 300, 41, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        kind = rng.choice(["accum", "accum", "accum", "four", "four", "four", "pack"])
        d = rng.choice([32, 64, 64, 128])
        dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
        c = _case(None, kind, dtype, _log_int(rng, 1, 128), rng.randint(1, 16), rng.choice([1, 1, 2, 3, 4, 5, 8, 12]), d, _log_int(rng, 13, 2048),
                  _log_int(rng, 1, 8192), 0, 0, rule=rng.choice(["accum", "learned"]) if kind == "four" else "accum",
                  decay=rng.choice([1.0, 1.0, 0.9, 0.5, 0.0]), sink=rng.choice([0, 0, 1, 4]), K=rng.choice([3, 5, 7, 13]), ragged=rng.random() < 0.3)
        if dtype == "f32":
            c["B"], c["R"] = min(c["B"], 8), min(c["R"], 1024)
        c["n"] = _log_int(rng, 2, c["W"]) if rng.random() < 0.15 else c["W"] + _log_int(rng, 1, 3 * c["R"] + 2)
        out = max(0, c["n"] - c["W"])
        c["cnt"] = min(c["R"], out)
        c["sink"] = min(c["sink"], c["R"], c["cnt"])
        if kind != "pack":
            c["steps"] = _log_int(rng, 1, 4) if kind == "accum" else _log_int(rng, 2, 16)
        if work(c)["bytes"] <= most:
            return c


# ---- where things stand in the caches (lte.h) ----------------------------------------------------------------------------


def _up(x, n):
    return (x + n - 1) // n * n


def _blocks(c, size):
    return torch.zeros(HEADER + c["B"] * c["H"] * size, dtype=torch.uint8, device="cuda")


def _ordinary(c):
    """Offsets in a head's block of an ordinary cache: keys, values, scores, positions, counters, its size, allocated rows."""
    d, e, rows = c["d"], DTYPES[c["dtype"]][2], c["W"] + c["R"]
    alloc = 256 if c["dtype"] == "bf16" and d == 64 and rows <= 256 else rows
    v = alloc * d * e
    z = 2 * v
    p = z + 4 * rows
    m = p + 4 * c["R"]
    return 0, v, z, p, m, _up(m + 16, 256), alloc


def _four(c):
    """The same for a cache in 4 bits: key codes, value codes, key and value parameters, scores, positions, counters, size."""
    d, rows = c["d"], c["W"] + c["R"]
    at, off = [], 0
    for size in (rows * d // 2, rows * d // 2, rows * d // 8, rows * d // 8, 4 * rows, 4 * c["R"], 16):
        at.append(off)
        off = _up(off + size, 16)
    return at + [_up(off, 256)]


def _at(buf, size, off, n, dtype):
    """n values of a type at an offset of every head's block."""
    e = torch.empty((), dtype=dtype).element_size()
    return buf[HEADER:].view(-1, size)[:, off:off + n * e].view(dtype)


def _ordinary_views(c, buf):
    k, v, z, p, m, size, alloc = _ordinary(c)
    dt, rows, d = DTYPES[c["dtype"]][0], c["W"] + c["R"], c["d"]
    return {"keys": _at(buf, size, k, alloc * d, dt), "values": _at(buf, size, v, alloc * d, dt), "scores": _at(buf, size, z, rows, torch.float32),
            "positions": _at(buf, size, p, c["R"], torch.int32), "counters": _at(buf, size, m, 4, torch.int32)}


def _four_views(c, buf):
    k, v, kp, vp, z, p, m, size = _four(c)
    rows, d = c["W"] + c["R"], c["d"]
    return {"kcodes": _at(buf, size, k, rows * d // 2, torch.uint8), "vcodes": _at(buf, size, v, rows * d // 2, torch.uint8),
            "kpar": _at(buf, size, kp, rows * d // 16, torch.bfloat16), "vpar": _at(buf, size, vp, rows * d // 16, torch.bfloat16),
            "scores": _at(buf, size, z, rows, torch.float32), "positions": _at(buf, size, p, c["R"], torch.int32),
            "counters": _at(buf, size, m, 4, torch.int32)}


def _element_order(c):
    """[rows, d] places of an ordinary cache's elements in a head's block (None: in order): short bf16 caches are swizzled."""
    rows, d = c["W"] + c["R"], c["d"]
    if not (c["dtype"] == "bf16" and d == 64 and rows <= 256):
        return None
    r, ch = torch.arange(rows, device="cuda")[:, None], torch.arange(d, device="cuda")[None, :]
    return r * d + ((((ch >> 3) ^ (r & 7)) << 3) | (ch & 7))


def _nibble_order(c, values):
    """[d] channel of every nibble of a row in 4 bits, in memory order (low nibble of a byte first)."""
    d = c["d"]
    groups, per = d // GROUP, 4 if values else 8
    nib = torch.arange(d, device="cuda")
    unit, i = nib // per, nib % per
    return (unit % groups) * GROUP + (unit // groups) * per + i


def _quantise(x):
    """Rows [..., d] -> codes [..., d] (0..15), step and zero [..., d / 32] in bf16."""
    g = x.float().reshape(*x.shape[:-1], -1, GROUP)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    step, zero = ((hi - lo) / 15).to(torch.bfloat16), lo.to(torch.bfloat16)
    bad = ~(torch.isfinite(step) & torch.isfinite(zero))
    s, z = step.float(), zero.float()
    codes = torch.where(bad | (s == 0), 0.0, ((g - z) / torch.where(s == 0, 1.0, s)).round().clamp(0, 15))
    nan = torch.full_like(step, float("nan"))
    return codes.reshape(x.shape).to(torch.uint8), torch.where(bad, nan, step)[..., 0], torch.where(bad, nan, zero)[..., 0]


def _to_bytes(codes, order):
    """Codes [..., d] -> bytes [..., d / 2]."""
    nib = codes[..., order]
    return nib[..., 0::2] | (nib[..., 1::2] << 4)


def _from_bytes(b, order, par):
    """Bytes [..., d / 2] and parameters [..., d / 16] -> values [..., d] in 32 bits."""
    nib = torch.stack([b & 15, b >> 4], dim=-1).flatten(-2)
    codes = torch.empty_like(nib)
    codes[..., order] = nib
    p = par.float().reshape(*par.shape[:-1], -1, 2)
    g = codes.float().reshape(*codes.shape[:-1], -1, GROUP)
    return (p[..., 1:] + g * p[..., :1]).reshape(codes.shape)


def _put_ordinary(c, view, order, rows):
    """Rows [heads, W + R, d] into the keys or values of an ordinary cache."""
    if order is None:
        view.copy_(rows.reshape(view.shape))
    else:
        view.zero_()
        view[:, order.reshape(-1)] = rows.reshape(rows.shape[0], -1).to(view.dtype)


def _get_ordinary(c, view, order):
    rows = c["W"] + c["R"]
    return (view[:, :rows * c["d"]] if order is None else view[:, order.reshape(-1)]).reshape(-1, rows, c["d"])


# ---- inputs -----------------------------------------------------------------------------------------------------------


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    B, H, G, d, W, R, n = (c[x] for x in ("B", "H", "G", "d", "W", "R", "n"))
    heads, rows, dt = B * H, W + R, DTYPES[c["dtype"]][0]

    def normal(*size, scale=1.0):
        return (torch.randn(size, generator=g, device=dev) * scale).to(dt)

    def uniform(*size):
        return torch.rand(size, generator=g, device=dev)

    # what n tokens have left: the ring's newest rows, and pool entries from all over the sequence
    out = max(0, n - W)
    cnt = torch.full((heads,), min(c["cnt"], R, out), device=dev)
    if c["ragged"] and out:
        cnt = (c["sink"] + uniform(heads) * (cnt + 1 - c["sink"])).long().minimum(cnt)
    j = torch.arange(R, device=dev)
    used = torch.cat([(torch.arange(W, device=dev) < n).expand(heads, W), j < cnt[:, None]], dim=1)
    each = max(1, out // max(1, min(c["cnt"], out)))                 # every entry from a stretch of its own
    pos = j * each + (uniform(heads, R) * each).long()
    pos[:, :c["sink"]] = j[:c["sink"]]
    k, v = normal(heads, rows, d, scale=d ** -0.25), normal(heads, rows, d)
    k, v = torch.where(used[..., None], k, 0), torch.where(used[..., None], v, 0)
    if c["rule"] == "accum":
        # attention received so far: a few tokens much, most little
        score = (1.5 * torch.randn((heads, rows), generator=g, device=dev)).exp()
    else:
        # logits of a trained scorer: what is in the pool has passed the threshold; the newest tokens have no logit yet
        score = 1.5 * torch.randn((heads, rows), generator=g, device=dev)
        score[:, W:] = score[:, W:].abs() + 1e-3
        for t in range(max(0, n - c["K"] // 2), n):
            score[:, t % W] = -float("inf")
    score = torch.where(used, score, -float("inf"))

    st = {"c": c, "order": _element_order(c), "cache": _blocks(c, _ordinary(c)[5])}
    st["views"] = w = _ordinary_views(c, st["cache"])
    if c["kind"] == "four":
        st["cache4"] = _blocks(c, _four(c)[7])
        st["views4"] = w = _four_views(c, st["cache4"])
        for x, name in ((k, "k"), (v, "v")):
            codes, step, zero = _quantise(x)
            w[name + "codes"].copy_(_to_bytes(codes, _nibble_order(c, name == "v")).flatten(1))
            w[name + "par"].copy_(torch.stack([step, zero], dim=-1).flatten(1))
    else:
        _put_ordinary(c, w["keys"], st["order"], k)
        _put_ordinary(c, w["values"], st["order"], v)
        if c["kind"] == "pack":
            st["cache4"] = _blocks(c, _four(c)[7])
            st["views4"] = _four_views(c, st["cache4"])
            st["back"] = torch.zeros_like(st["cache"])
            st["back_views"] = _ordinary_views(c, st["back"])
    w["scores"].copy_(score)
    w["positions"].copy_(torch.where(j < cnt[:, None], pos, 0))
    w["counters"][:, 0] = n
    w["counters"][:, 1] = cnt
    if c["kind"] != "pack":
        steps = c["steps"]
        st["tokens"] = list(zip(normal(steps, B, H * G, d, scale=2.0 * d ** -0.25), normal(steps, B, H, d, scale=d ** -0.25), normal(steps, B, H, d)))
    if c["rule"] == "learned":
        st["w"], st["bias"] = torch.randn((H, c["K"], 2 * d), generator=g, device=dev) * 0.05, torch.randn((H,), generator=g, device=dev) * 0.1
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------


def run(state):
    return _calls(state) if own else _plain(state)


def _calls(st):
    from paper_2510_20787_b200 import lte
    c = st["c"]
    s = lte.shape(c["B"], c["H"], 0, c["d"], c["W"], c["R"], DTYPES[c["dtype"]][1], sink=c["sink"], group=c["G"])
    if c["kind"] == "pack":
        lte.lte_cache4_pack(s, st["cache"], cache4=st["cache4"])
        lte.lte_cache4_unpack(s, st["cache4"], cache=st["back"])
        return st["back_views"]
    if c["kind"] == "accum":
        got = [lte.lte_attn_decode_accum(s, st["cache"], q, k, v, decay=c["decay"]) for q, k, v in st["tokens"]]
    elif c["rule"] == "accum":
        got = [lte.lte_attn_decode4_accum(s, st["cache4"], q, k, v, decay=c["decay"]) for q, k, v in st["tokens"]]
    else:
        conv = lte.conv(st["w"], st["bias"])
        got = [lte.lte_attn_decode4(s, conv, st["cache4"], q, k, v) for q, k, v in st["tokens"]]
    if c["kind"] == "four":
        lte.lte_cache4_unpack(s, st["cache4"], cache=st["cache"])
    return dict(st["views"], o=[x for x, _ in got], lse=[x for _, x in got])


def _plain(st):
    c = st["c"]
    kord, vord = _nibble_order(c, False), _nibble_order(c, True)
    if c["kind"] == "pack":
        a, b, w = st["views"], st["views4"], st["back_views"]
        for name, full, order in (("k", "keys", kord), ("v", "values", vord)):
            codes, step, zero = _quantise(_get_ordinary(c, a[full], st["order"]))
            b[name + "codes"].copy_(_to_bytes(codes, order).flatten(1))
            b[name + "par"].copy_(torch.stack([step, zero], dim=-1).flatten(1))
        for name in ("scores", "positions", "counters"):
            b[name].copy_(a[name])
        return _plain_unpack(c, b, w, st["order"], kord, vord)
    got = [_plain_step(st, q, k, v, kord, vord) for q, k, v in st["tokens"]]
    if c["kind"] == "four":
        _plain_unpack(c, st["views4"], st["views"], st["order"], kord, vord)
    return dict(st["views"], o=[x for x, _ in got], lse=[x for _, x in got])


def _plain_rows(c, w4, name, order):
    heads, rows, d = w4["scores"].shape[0], c["W"] + c["R"], c["d"]
    return _from_bytes(w4[name + "codes"].reshape(heads, rows, d // 2), order, w4[name + "par"].reshape(heads, rows, d // 16))


def _plain_unpack(c, w4, w, eorder, kord, vord):
    _put_ordinary(c, w["keys"], eorder, _plain_rows(c, w4, "k", kord))
    _put_ordinary(c, w["values"], eorder, _plain_rows(c, w4, "v", vord))
    for name in ("scores", "positions", "counters"):
        w[name].copy_(w4[name])
    return w


def _plain_step(st, q1, k1, v1, kord, vord):
    c = st["c"]
    four = c["kind"] == "four"
    w = st["views4"] if four else st["views"]
    B, H, G, d, W, R, sink = (c[x] for x in ("B", "H", "G", "d", "W", "R", "sink"))
    heads, rows = B * H, W + R
    if four:
        keys, values = _plain_rows(c, w, "k", kord), _plain_rows(c, w, "v", vord)
    else:
        keys, values = _get_ordinary(c, w["keys"], st["order"]).float(), _get_ordinary(c, w["values"], st["order"]).float()
    kn, vn, q = k1.reshape(heads, d).float(), v1.reshape(heads, d).float(), q1.reshape(heads, G, d).float()
    score, pos = w["scores"], w["positions"].long()
    n, cnt = w["counters"][:, 0].long(), w["counters"][:, 1].long()
    slot, p = n % W, n - W
    head, j = torch.arange(heads, device=q.device), torch.arange(R, device=q.device)

    # the token that leaves the window
    leaving = score[head, slot]
    wants = (p >= 0) & ((p < sink) | (leaving > 0) if c["rule"] == "learned" else p >= 0)
    may_go = (j < cnt[:, None]) & (pos >= sink)
    least = torch.where(may_go, score[:, W:], float("inf")).amin(1)
    worst = torch.where(may_go & (score[:, W:] == least[:, None]), pos, -1).argmax(1)
    room = cnt < R
    dst = torch.where(wants & room, cnt, torch.where(wants & ~room & (p >= sink) & may_go.any(1) & (leaving > least), worst, -1))

    # attention over the ring, the pool and the incoming token
    r = torch.arange(W, device=q.device)
    ring = (r < n[:, None]) & ~((r == slot[:, None]) & (p >= 0)[:, None] & (dst < 0)[:, None])
    seen = torch.cat([ring, (j < cnt[:, None]) & (j != dst[:, None])], dim=1)
    scale = d ** -0.5
    x = torch.cat([(q @ keys.transpose(1, 2)) * scale, (q * kn[:, None]).sum(-1, keepdim=True) * scale], dim=2)
    x = torch.where(torch.cat([seen, torch.ones_like(seen[:, :1])], dim=1)[:, None], x, -float("inf"))
    top = x.amax(-1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(-1, keepdim=True)
    weight = e / total
    o = weight[..., :rows] @ values + weight[..., rows:] * vn[:, None]
    lse = (top + total.log())[..., 0]

    # scores
    if c["rule"] == "accum":
        got = weight.sum(1)
        new = torch.where(seen, c["decay"] * score + got[:, :rows], score)
        moved, fresh = new[head, slot], got[:, rows]
    else:
        new, moved, fresh = score.clone(), leaving, torch.full_like(leaving, -float("inf"))

    # the row that leaves moves into the pool, the incoming one takes its place
    to = W + dst.clamp(min=0)
    takes = dst >= 0
    new[head, to] = torch.where(takes, moved, new[head, to])
    new[head, slot] = fresh
    if c["rule"] == "learned":
        K = c["K"]
        target = n - K // 2
        taps = target[:, None] + torch.arange(K, device=q.device) - K // 2
        kx = torch.where((taps == n[:, None])[..., None], kn[:, None], keys[head[:, None], taps % W])
        vx = torch.where((taps == n[:, None])[..., None], vn[:, None], values[head[:, None], taps % W])
        each = (torch.cat([kx, vx], dim=-1) * st["w"].repeat(B, 1, 1)).sum(-1)
        z = torch.where(taps >= 0, each, 0).sum(1) + st["bias"].repeat(B)
        at = target % W
        new[head, at] = torch.where(target >= 0, z, new[head, at])
    w["scores"].copy_(new)
    newpos = w["positions"].clone()
    newpos[head, to - W] = torch.where(takes, p, pos[head, to - W]).int()
    w["positions"].copy_(newpos)
    w["counters"][:, 0] += 1
    w["counters"][:, 1] += (wants & room).int()
    if four:
        for x, name, order in ((kn, "k", kord), (vn, "v", vord)):
            codes, step, zero = _quantise(x)
            _plain_move(w[name + "codes"].unflatten(1, (rows, d // 2)), _to_bytes(codes, order), head, slot, to, takes)
            _plain_move(w[name + "par"].unflatten(1, (rows, d // 16)), torch.stack([step, zero], dim=-1).flatten(1), head, slot, to, takes)
    elif st["order"] is None:
        _plain_move(w["keys"].unflatten(1, (rows, d)), k1.reshape(heads, d), head, slot, to, takes)
        _plain_move(w["values"].unflatten(1, (rows, d)), v1.reshape(heads, d), head, slot, to, takes)
    else:
        a, b = st["order"][slot], st["order"][to]
        for name, x in (("keys", k1), ("values", v1)):
            view = w[name]
            view[head[:, None], b] = torch.where(takes[:, None], view[head[:, None], a], view[head[:, None], b])
            view[head[:, None], a] = x.reshape(heads, d)
    return o.reshape(B, H * G, d).to(q1.dtype), lse.reshape(B, H * G)


def _plain_move(view, x, head, slot, to, takes):
    view[head, to] = torch.where(takes[:, None], view[head, slot], view[head, to])
    view[head, slot] = x


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def exact(case, seed):
    """Head by head where the pool decides, all heads at once where they attend; 4-bit rows by their rule, which is stated in 32 bits."""
    c = case
    if c["B"] * c["H"] * c["steps"] > 40000:
        return None
    st = prepare(case, seed)
    B, H, G, d, W, R, sink = (c[x] for x in ("B", "H", "G", "d", "W", "R", "sink"))
    heads, rows = B * H, W + R
    w = st["views4"] if c["kind"] == "four" else st["views"]
    if c["kind"] == "four":
        K64 = _exact_rows(w["kcodes"], w["kpar"], rows, d, 8)
        V64 = _exact_rows(w["vcodes"], w["vpar"], rows, d, 4)
    else:
        perm = None
        if st["order"] is not None:
            perm = np.array([[r * d + ((((ch // 8) ^ (r % 8)) * 8) + ch % 8) for ch in range(d)] for r in range(rows)])
        K64, V64 = (_exact_ordinary(w[x], perm, rows, d) for x in ("keys", "values"))
    score, pos = w["scores"].cpu().numpy().astype(np.float64), w["positions"].cpu().numpy().astype(np.int64)
    count = w["counters"].cpu().numpy().astype(np.int64)
    if c["kind"] == "pack":
        K64, V64 = _exact_held(K64), _exact_held(V64)
        return _exact_out(c, K64, V64, score, pos, count)
    os, lses = [], []
    for q1, k1, v1 in st["tokens"]:
        q, kn, vn = q1.double().reshape(heads, G, d), k1.double().reshape(heads, 1, d), v1.double().reshape(heads, 1, d)
        slots, dsts = np.empty(heads, np.int64), np.full(heads, -1, np.int64)
        hide = np.zeros((heads, rows + 1), bool)
        for h in range(heads):
            n, m = count[h, 0], count[h, 1]
            p, slot = n - W, n % W
            slots[h] = slot
            hide[h, min(n, W):W] = True
            hide[h, W + m:rows] = True
            if p < 0:
                continue
            a = score[h, slot]
            if R > 0 and (c["rule"] == "accum" or p < sink or a > 0):
                if m < R:
                    dsts[h] = m
                elif p >= sink:
                    some = np.flatnonzero(pos[h] >= sink)
                    if some.size:
                        low = score[h, W + some].min()
                        tied = some[score[h, W + some] == low]
                        if a > low:
                            dsts[h] = tied[np.argmax(pos[h, tied])]
            if dsts[h] < 0:
                hide[h, slot] = True
            elif dsts[h] < m:
                hide[h, W + dsts[h]] = True
        x = torch.cat([K64, kn], dim=1) @ q.transpose(1, 2) / math.sqrt(d)
        x.masked_fill_(torch.from_numpy(hide).cuda()[..., None], -float("inf"))
        lse = torch.logsumexp(x, dim=1)
        weight = (x - lse[:, None]).exp()
        os.append((weight.transpose(1, 2) @ torch.cat([V64, vn], dim=1)).reshape(B, H * G, d))
        lses.append(lse.reshape(B, H * G))
        got = weight.sum(-1).cpu().numpy()
        if c["rule"] == "learned":
            wt, bias = st["w"].double(), st["bias"].double().cpu().numpy()
            K = c["K"]
            n = int(count[0, 0])                                     # the same in every head
            z = torch.zeros(heads, dtype=torch.float64, device="cuda")
            for t in range(K):
                tok = n - K // 2 + t - K // 2
                if tok >= 0:
                    kr, vr = (kn[:, 0], vn[:, 0]) if tok == n else (K64[:, tok % W], V64[:, tok % W])
                    z += (torch.cat([kr, vr], dim=1).reshape(B, H, 2 * d) * wt[:, t]).sum(-1).reshape(heads)
            z = z.cpu().numpy() + np.tile(bias, B)
        ks, vs = _exact_held(kn)[:, 0] if c["kind"] == "four" else kn[:, 0], _exact_held(vn)[:, 0] if c["kind"] == "four" else vn[:, 0]
        if c["rule"] == "accum":
            score = np.where(hide[:, :rows], score, c["decay"] * score + got[:, :rows])
        took = np.flatnonzero(dsts >= 0)
        i, a, b = torch.from_numpy(took).cuda(), torch.from_numpy(slots[took]).cuda(), torch.from_numpy(W + dsts[took]).cuda()
        K64[i, b], V64[i, b] = K64[i, a], V64[i, a]
        score[took, W + dsts[took]] = score[took, slots[took]]
        pos[took, dsts[took]] = count[took, 0] - W
        every = np.arange(heads)
        K64[torch.from_numpy(every).cuda(), torch.from_numpy(slots).cuda()] = ks
        V64[torch.from_numpy(every).cuda(), torch.from_numpy(slots).cuda()] = vs
        score[every, slots] = got[:, rows] if c["rule"] == "accum" else -np.inf
        if c["rule"] == "learned" and n - c["K"] // 2 >= 0:
            score[:, (n - c["K"] // 2) % W] = z
        count[took, 1] += dsts[took] >= count[took, 1]
        count[:, 0] += 1
    return dict(_exact_out(c, K64, V64, score, pos, count), o=os, lse=lses)


def _exact_ordinary(view, perm, rows, d):
    flat = view.double()
    return (flat[:, torch.from_numpy(perm.reshape(-1)).cuda()] if perm is not None else flat[:, :rows * d]).reshape(-1, rows, d).clone()


def _exact_rows(codes, par, rows, d, per):
    """4-bit rows as the values they stand for: unit u of ``per`` nibbles holds channels of group u mod (d / 32)."""
    b = codes.cpu().numpy().reshape(-1, rows, d // 2)
    nib = np.empty(b.shape[:2] + (d,), np.float64)
    nib[..., 0::2], nib[..., 1::2] = b % 16, b // 16
    groups = d // GROUP
    a = nib.reshape(b.shape[:2] + (GROUP // per, groups, per)).transpose(0, 1, 3, 2, 4).reshape(b.shape[:2] + (groups, GROUP))
    p = par.double().cpu().numpy().reshape(b.shape[:2] + (groups, 2))
    return torch.from_numpy((a * p[..., :1] + p[..., 1:]).reshape(b.shape[:2] + (d,))).cuda()


def _exact_held(x):
    """Rows as a 4-bit cache holds them: the codes by their rule (fp32 arithmetic, parameters in bf16), the values from them in 64 bits."""
    a = x.float().cpu().numpy().reshape(-1, GROUP)
    lo, hi = a.min(1), a.max(1)
    bf = lambda t: torch.from_numpy(t).to(torch.bfloat16).float().numpy()  # noqa: E731
    step, zero = bf((hi - lo) / np.float32(15)), bf(lo)
    some = step > 0
    code = np.where(some[:, None], np.clip(np.rint((a - zero[:, None]) / np.where(some, step, np.float32(1))[:, None]), 0, 15), 0)
    out = zero[:, None].astype(np.float64) + code.astype(np.float64) * step[:, None].astype(np.float64)
    return torch.from_numpy(out.reshape(x.shape)).to(x.device)


def _exact_out(c, K64, V64, score, pos, count):
    """As run() lays the state out."""
    heads, rows, d = K64.shape
    alloc = _ordinary(c)[6]
    out = {}
    for name, x in (("keys", K64), ("values", V64)):
        if alloc != rows or _element_order(c) is not None:
            y = torch.zeros((heads, alloc, d // 8, 8), dtype=torch.float64, device=x.device)
            for piece in range(d // 8):
                for k in range(8):
                    r = torch.arange(k, rows, 8, device=x.device)
                    y[:, r, piece ^ k] = x[:, r, piece * 8:piece * 8 + 8]
            x = y
        out[name] = x.reshape(heads, -1)
    return dict(out, scores=torch.from_numpy(score), positions=torch.from_numpy(pos.astype(np.int32)), counters=torch.from_numpy(count.astype(np.int32)))


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------


def work(case):
    """Rows in use and their scores read once, what changes written once; multiply-adds of the logits and the output."""
    c = case
    e = DTYPES[c["dtype"]][2]
    B, H, G, d, W, R = (c[x] for x in ("B", "H", "G", "d", "W", "R"))
    heads = B * H
    held = min(c["cnt"], R, max(0, c["n"] - W)) / (2 if c["ragged"] else 1)
    used = min(c["n"], W) + held
    full, four = 2 * d * e, 2 * (d // 2 + d // 8)                    # bytes of a key and a value
    small = 4 * (W + R) + 4 * R + 16
    if c["kind"] == "pack":
        return {"bytes": 2.0 * heads * (used * (full + four) + 2 * small), "flops": 0.0}
    row = four if c["kind"] == "four" else full
    scores = (8 * used if c["rule"] == "accum" else 4 * held) + 4 * held
    step = heads * (used * row + scores + full + row + G * (2 * d * e + 4))
    flops = heads * 4.0 * d * G * used
    if c["rule"] == "learned":
        step += 4 * H * (c["K"] * 2 * d + 1)
        flops += heads * 4.0 * c["K"] * d
    bytes_ = c["steps"] * step
    if c["kind"] == "four":
        bytes_ += heads * (used * (full + four) + 2 * small)
    return {"bytes": float(bytes_), "flops": float(c["steps"] * flops)}
