"""One decode step over a cache that evicts by accumulated attention or holds 4 bits, in 64 bits, from a cache's bytes as lte.h lays
them out; and how far fp32 arithmetic may be from it.

The step starts from the bytes that the kernel starts from, so that a decision (an ordering of fp32 scores) is the same one.
"""
import numpy as np
import torch

EPS = 2.0 ** -24


def up(x, n):
    return (x + n - 1) // n * n


class Layout:
    """Views of every head's parts in a cache (a CUDA or CPU byte tensor)."""

    def __init__(self, s, four):
        self.s, self.four, self.rows = s, four, s.W + s.R
        self.esz = 2 if s.dtype == 1 else 4
        if four:
            sizes = [self.rows * s.d // 2, self.rows * s.d // 2, self.rows * s.d // 8, self.rows * s.d // 8, 4 * self.rows, 4 * s.R, 16]
            names, align = ["k", "v", "kpar", "vpar", "score", "pos", "count"], 16
            self.swizzled = False
        else:
            self.swizzled = s.dtype == 1 and s.d == 64 and self.rows <= 256
            alloc = 256 if self.swizzled else self.rows
            sizes = [alloc * s.d * self.esz, alloc * s.d * self.esz, 4 * self.rows, 4 * s.R, 16]
            names, align = ["k", "v", "score", "pos", "count"], 1
        off, self.at = 0, {}
        for name, size in zip(names, sizes):
            self.at[name] = (off, off + size)
            off = up(off + size, align)
        self.stride = up(off, 256)

    def part(self, cache, name, dtype, heads=slice(None)):
        a, b = self.at[name]
        return cache[256:].view(-1, self.stride)[heads, a:b].contiguous().view(dtype)

    def rows_of(self, cache, name, heads=slice(None)):
        """Keys or values as the cache holds them: float64 [heads, W + R, d]."""
        s = self.s
        if self.four:
            b = self.part(cache, name, torch.uint8, heads).cpu().numpy().reshape(-1, self.rows, s.d // 2)
            par = self.part(cache, name + "par", torch.bfloat16, heads).double().cpu().numpy().reshape(-1, self.rows, s.d // 32, 2)
            out = np.empty((b.shape[0], self.rows, s.d))
            per = 8 if name == "k" else 4
            for x in range(s.d):                               # nibble x of a row
                unit, i = divmod(x, per)
                g, t = unit % (s.d // 32), unit // (s.d // 32)
                code = (b[..., x // 2] >> (4 * (x % 2))) & 15
                out[..., g * 32 + t * per + i] = par[..., g, 1] + code * par[..., g, 0]
            return out
        x = self.part(cache, name, torch.bfloat16 if self.esz == 2 else torch.float32, heads).double().cpu().numpy()
        x = x.reshape(x.shape[0], -1, s.d)
        if self.swizzled:
            y = np.empty_like(x)
            for r in range(x.shape[1]):
                for c in range(8):
                    y[:, r, 8 * c:8 * c + 8] = x[:, r, 8 * (c ^ (r & 7)):8 * (c ^ (r & 7)) + 8]
            x = y
        return x[:, :self.rows]

    def state(self, cache, heads=slice(None)):
        count = self.part(cache, "count", torch.int32, heads).cpu().numpy().astype(np.int64)
        return {"k": self.rows_of(cache, "k", heads), "v": self.rows_of(cache, "v", heads),
                "score": self.part(cache, "score", torch.float32, heads).double().cpu().numpy(),
                "pos": self.part(cache, "pos", torch.int32, heads).cpu().numpy().astype(np.int64).reshape(len(count), self.s.R), "count": count}


def four(x):
    """Rows [..., d] as 4 bits hold them (the rule's arithmetic is fp32), with step and zero per channel."""
    x = np.asarray(x, np.float32)
    g = x.reshape(-1, 32)
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16).float().numpy()  # noqa: E731
    with np.errstate(all="ignore"):
        step, zero = bf((g.max(1) - g.min(1)) * (np.float32(1) / np.float32(15))), bf(g.min(1))
        bad = ~(np.isfinite(step) & np.isfinite(zero) & np.isfinite(g).all(1))
        code = np.clip(np.rint((g - zero[:, None]) / np.where(step > 0, step, 1)[:, None]), 0, 15)
    code = np.where((step > 0)[:, None] & ~bad[:, None], code, 0)
    with np.errstate(all="ignore"):
        val = np.where(bad[:, None], np.nan, zero[:, None].astype(np.float64) + code * step[:, None].astype(np.float64))
    per = lambda a: np.repeat(a[:, None], 32, axis=1).reshape(x.shape).astype(np.float64)  # noqa: E731
    return val.reshape(x.shape), per(step), per(zero)


def step(s, lay, before, q1, k1, v1, accum, decay=1.0, w=None, bias=None, which=None):
    """State after one step, o, lse in 64 bits, and bounds of the error of each: {"o", "lse", "score"}.  which: the heads that `before`, q1, k1, v1
    are of (all)."""
    st = {n: a.copy() for n, a in before.items()}
    which = list(range(s.B * s.H)) if which is None else which
    heads, W, R, d, G = len(which), s.W, s.R, s.d, max(1, s.group)
    scale = s.softmax_scale if s.softmax_scale > 0 else 1.0 / np.sqrt(d)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    q, kn, vn = f(q1).reshape(heads, G, d), f(k1).reshape(heads, d), f(v1).reshape(heads, d)
    rounded = s.dtype == 1
    o, lse = np.empty((heads, G, d)), np.empty((heads, G))
    bound = {"o": np.empty((heads, G, d)), "lse": np.empty((heads, G)), "score": np.zeros((heads, W + R))}
    for h in range(heads):
        n, cnt = st["count"][h, 0], st["count"][h, 1]
        p, slot = n - W, n % W
        sc, pos = st["score"][h], st["pos"][h]
        rows = {r: r for r in range(min(n, W))}                # row -> where its score goes
        rows.update({W + m: W + m for m in range(cnt)})
        taken = -1
        if p >= 0:
            want = R > 0 and (accum or p < s.sink or sc[slot] > np.log(s.tau) - np.log1p(-s.tau))
            if want and cnt < R:
                taken = cnt
                st["count"][h, 1] += 1
            elif want and p >= s.sink:
                may = [m for m in range(cnt) if pos[m] >= s.sink]
                if may:
                    worst = min(may, key=lambda m: (sc[W + m], -pos[m]))
                    if sc[slot] > sc[W + worst]:
                        taken = worst
            if taken < 0:
                del rows[slot]
            else:
                rows.pop(W + taken, None)
                rows[slot] = W + taken
        idx = np.array(sorted(rows), dtype=np.int64)
        K = np.concatenate([st["k"][h, idx], kn[h:h + 1]])
        V = np.concatenate([st["v"][h, idx], vn[h:h + 1]])
        # magnitudes that fp32 rounds: products, and for 4 bits (code + 16) step + (zero - 16 step), each at most 48 step + |zero|
        mk, mv = np.abs(K), np.abs(V)
        if lay.four:
            for m, name in ((mk, "k"), (mv, "v")):
                par = before[name + "mag"][h, idx]
                m[:-1] = np.maximum(m[:-1], par)
        with np.errstate(all="ignore"):
            x = (q[h] @ K.T) * scale
            top = x.max(1, keepdims=True)
            lse[h] = top[:, 0] + np.log(np.exp(x - top).sum(1))
            wt = np.exp(x - lse[h][:, None])
            o[h] = wt @ V
        m = len(idx) + 1
        ex = EPS * (d + 8) * ((np.abs(q[h]) @ mk.T) * scale).max(1)
        ew = 2 * ex + 2.0 ** -21 + EPS * (4 * np.maximum(0, (top - x)[wt > 1e-30].max(initial=0)) + m + 16)
        bound["lse"][h] = ex + EPS * (m + 16 + 8 * np.abs(lse[h]))
        # (bf16 calls multiply a weight as the sum of two bf16 numbers: 2^-16 of every product; over 4 bits a weight times its row's step is
        # rounded to fp16, 2^-12 of products with codes, w code step <= w 15 step <= w mv 15 / 48)
        bound["o"][h] = ew[:, None] * (wt @ np.abs(V)) * 2 + (EPS * (m + 16) + (2.0 ** -12 * 15 / 48 if rounded and lay.four else 2.0 ** -16 if rounded else 0)) * (wt @ mv) + (2.0 ** -8 if rounded else EPS) * np.abs(o[h])
        if accum:
            got = wt.sum(0)
            new = {rows[r]: decay * sc[r] + got[i] if decay else got[i] for i, r in enumerate(idx)}
            err = {rows[r]: (ew[:, None] * wt).sum(0)[i] + EPS * (G + 4) * (abs(decay * sc[r]) + got[i]) for i, r in enumerate(idx)}
            for r in new:
                st["score"][h, r], bound["score"][h, r] = new[r], err[r]
            st["score"][h, slot], bound["score"][h, slot] = got[-1], (ew[:, None] * wt).sum(0)[-1] + EPS * (G + 4) * got[-1]
        else:
            if taken >= 0:
                st["score"][h, W + taken] = sc[slot]
            st["score"][h, slot] = -np.inf
            taps = w.shape[1]
            j = n - taps // 2
            if j >= 0:
                z, mag, hw = 0.0 if bias is None else float(bias[which[h] % s.H]), 0.0, which[h] % s.H
                for t in range(taps):
                    tok = j + t - taps // 2
                    if tok >= 0:
                        kr, vr = (kn[h], vn[h]) if tok == n else (before["k"][h, tok % W], before["v"][h, tok % W])
                        z += w[hw, t, :d] @ kr + w[hw, t, d:] @ vr
                        mag += np.abs(w[hw, t, :d]) @ np.abs(kr) + np.abs(w[hw, t, d:]) @ np.abs(vr)
                st["score"][h, j % W] = z
                bound["score"][h, j % W] = EPS * (2 * d * taps + taps + 2) * (mag + abs(z))
        if taken >= 0:
            st["k"][h, W + taken], st["v"][h, W + taken] = before["k"][h, slot], before["v"][h, slot]
            st["pos"][h, taken] = p
        st["k"][h, slot], st["v"][h, slot] = (four(kn[h])[0], four(vn[h])[0]) if lay.four else (kn[h], vn[h])
        st["count"][h, 0] += 1
    return st, o, lse, bound


def magnitudes(lay, cache, state, heads=slice(None)):
    """48 step + |zero| of every channel of a cache in 4 bits, for the bounds."""
    for name in ("k", "v"):
        par = lay.part(cache, name + "par", torch.bfloat16, heads).double().cpu().numpy().reshape(-1, lay.rows, lay.s.d // 32, 2)
        state[name + "mag"] = np.repeat(48 * par[..., 0] + np.abs(par[..., 1]), 32, axis=-1)
    return state


def check_step(s, lay, cache, q1, k1, v1, call, accum, decay=1.0, w=None, bias=None, which=None):
    """Runs `call` on the cache and holds what it leaves (in the heads `which`) to the step in 64 bits.  Returns o, lse of the call."""
    heads = slice(None) if which is None else torch.tensor(which, device=cache.device)
    of = lambda t, d: t.reshape(s.B * s.H, -1, d)[heads]  # noqa: E731
    before = lay.state(cache, heads)
    if lay.four:
        magnitudes(lay, cache, before, heads)
    want, o64, l64, bound = step(s, lay, before, of(q1, s.d), of(k1, s.d), of(v1, s.d), accum, decay, w, bias, which)
    o, lse = call()
    torch.cuda.synchronize()
    after = lay.state(cache, heads)
    assert np.array_equal(after["count"], want["count"]) and np.array_equal(after["pos"], want["pos"])
    assert np.array_equal(after["k"], want["k"], equal_nan=True) and np.array_equal(after["v"], want["v"], equal_nan=True)
    near("score", after["score"], want["score"], bound["score"])
    near("lse", of(lse, 1).double().cpu().numpy().reshape(l64.shape), l64, bound["lse"])
    near("o", of(o, s.d).double().cpu().numpy().reshape(o64.shape), o64, bound["o"])
    return o, lse


def near(name, got, want, bound):
    same = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), same) and np.array_equal(np.isnan(got), np.isnan(want)), name
    assert np.array_equal(got[~same & ~np.isnan(want)], want[~same & ~np.isnan(want)]), name
    off, most = np.abs(got[same] - want[same]), bound[same]
    assert bool((off <= most).all()), (name, float((off - most).max()), float((off / np.maximum(most, 1e-300)).max()))
