"""Attention and its gradient from their formulas in 64 bits, head by head on the CPU, and how far a
kernel that rounds as documented may be from them.  Test infrastructure only; nothing of the library.

A rounding to a type is off by at most half a step, u = eps / 2 of the value.  The bounds below add up,
entry by entry: probabilities (and their gradients) rounded once to the type, the result rounded once, and 32-bit
sums and exponentials."""
import math

import torch

STEP32 = 2.0 ** -24


def _docs(n, m, starts, k_starts, prefix):
    if starts is None:
        return [(0, n, 0, m, 0 if prefix is None else int(prefix[0]))]
    return [(starts[c], starts[c + 1], k_starts[c], k_starts[c + 1], 0 if prefix is None else prefix[c])
            for c in range(len(starts) - 1)]


def attention(Q, K, V, dO=None, scale=None, causal=False, cap=0.0, slopes=None, starts=None, k_starts=None, prefix=None):
    """Dict of O, lse and, with dO, dQ, dK, dV (float64; rows and keys outside the documents NaN), and for each a
    bound on what a kernel may be off, "O+" and so on."""
    eps = torch.finfo(Q.dtype).eps / 2
    tiny = 2.0 ** -25 if Q.dtype == torch.float16 else 2.0 ** -134  # half the smallest step of the type
    Q, K, V = (t.detach().double().cpu() for t in (Q, K, V))
    dO = None if dO is None else dO.detach().double().cpu()
    (n, hq, d), (m, hkv, _) = Q.shape, K.shape
    scale = d ** -0.5 if scale is None else scale
    if k_starts is None:
        k_starts = starts
    nan = float("nan")
    r = {"O": torch.full((n, hq, d), nan, dtype=torch.float64), "lse": torch.full((hq, n), nan, dtype=torch.float64)}
    r["O+"], r["lse+"] = torch.zeros_like(r["O"]), torch.zeros_like(r["lse"])
    if dO is not None:
        for name, like in (("dQ", Q), ("dK", K), ("dV", V)):
            r[name] = torch.full_like(like, nan)
            r[name + "+"] = torch.zeros_like(like)
    for q0, q1, k0, k1, pre in _docs(n, m, starts, k_starts, prefix):
        nq, nk = q1 - q0, k1 - k0
        p = torch.arange(nq)[:, None] + nk - nq
        j = torch.arange(nk)[None, :]
        seen = ((j <= p) | (j < pre)) if causal else torch.ones(nq, nk, dtype=torch.bool)
        if dO is not None:
            for name in ("dK", "dV"):
                r[name][k0:k1] = 0.0
        for h in range(hq):
            f = h * hkv // hq
            q, k, v = Q[q0:q1, h], K[k0:k1, f], V[k0:k1, f]
            u = scale * (q @ k.T)
            # 32 bits: the product, then the steps that make a score of it
            off = STEP32 * (d + 8) * scale * (q.abs() @ k.abs().T)
            s, steep = u, torch.ones_like(u)
            if cap:
                t = torch.tanh(u / cap)
                s, steep = cap * t, 1 - t * t
                off = off + 16 * STEP32 * cap
            if slopes is not None:
                far = float(slopes[h]) * (p - j).abs().double()
                s = s - far
                off = off + 4 * STEP32 * far
            off = off + 8 * STEP32 * (1 + s.abs())
            s = s.masked_fill(~seen, -math.inf)
            some = seen.any(1)
            lse = torch.logsumexp(s, 1) if nk else torch.full((nq,), -math.inf, dtype=torch.float64)
            P = torch.where(seen, torch.exp(s - lse[:, None]), torch.zeros_like(s))
            P[~some] = 0.0
            err = torch.where(seen, off, torch.zeros_like(off)).amax(1, keepdim=True) if nk else torch.zeros(nq, 1)
            err = 2 * err  # of a probability, relative: its own score and the log-sum
            O = P @ v
            r["O"][q0:q1, h], r["lse"][h, q0:q1] = O, lse
            # probabilities are at most 1 above a sum of at least 1: an absolute error of `tiny` each
            offO = (eps + 2 * err) * (P @ v.abs()) + tiny * (seen.double() @ v.abs()) + eps * O.abs() + tiny
            r["O+"][q0:q1, h] = 1.01 * offO
            r["lse+"][h, q0:q1] = err[:, 0] + 8 * STEP32 * torch.where(some, lse.abs(), torch.zeros_like(lse))
            if dO is None or not nk or not nq:
                if dO is not None:
                    r["dQ"][q0:q1, h] = 0.0
                continue
            g = dO[q0:q1, h]
            gv = g @ v.T
            D = (g * O).sum(1, keepdim=True)
            ds = P * (gv - D) * steep
            # of the difference: 32-bit products, and O as the forward pass has rounded it; of the cap's slope
            # the same error as of its score over the cap
            off_in = STEP32 * (d + 4) * (g.abs() @ v.abs().T + (g * O).abs().sum(1, keepdim=True)) + \
                (g.abs() * offO).sum(1, keepdim=True)
            off_ds = (eps + err + 8 * STEP32) * ds.abs() + P * off_in * steep + tiny
            if cap:
                off_ds = off_ds + P * (gv - D).abs() * (2 * off / cap + 16 * STEP32)
            off_ds = torch.where(seen, off_ds, torch.zeros_like(off_ds))
            off_P = torch.where(seen, (eps + err) * P + tiny, torch.zeros_like(P))
            r["dQ"][q0:q1, h] = scale * ds @ k
            r["dQ+"][q0:q1, h] = 1.01 * (scale * (off_ds + (nk + 4) * STEP32 * ds.abs()) @ k.abs() + eps * (scale * ds @ k).abs() + tiny)
            r["dK"][k0:k1, f] += scale * ds.T @ q
            r["dK+"][k0:k1, f] += 1.01 * (scale * (off_ds + (nq * hq + 4) * STEP32 * ds.abs()).T @ q.abs())
            r["dV"][k0:k1, f] += P.T @ g
            r["dV+"][k0:k1, f] += 1.01 * ((off_P + (nq * hq + 4) * STEP32 * P).T @ g.abs())
    if dO is not None:
        for name in ("dK", "dV"):
            r[name + "+"] += eps * r[name].abs() + tiny
    return r


def compare(name, got, r):
    """got against r[name] under r[name + "+"]; entries that r has as NaN are not looked at."""
    got, want, most = got.double().cpu(), r[name], r[name + "+"]
    look = ~torch.isnan(want)
    same = torch.where(torch.isinf(want), got == want, (got - want).abs() <= most)
    bad = look & ~same
    if bad.any():
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{name}: {int(bad.sum())} of {int(look.sum())} off, first at {at}: got {float(got[tuple(at)])}, "
                             f"want {float(want[tuple(at)])} within {float(most[tuple(at)])}")
    fine = look & torch.isfinite(want)
    return float(((got - want).abs()[fine] / most[fine].clamp(min=1e-300)).max()) if fine.any() else 0.0


# ---- the cache ------------------------------------------------------------------------------

def positive_codes(code):
    """The values of the codes without a sign, ascending."""
    if code == "int8":
        return torch.arange(128, dtype=torch.float64)
    return torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()


MOST = {"int8": 127.0, "e4m3": 448.0}


def nearest(y, code):
    """The codes' values nearest to 64-bit numbers, of two as near the one of even number; NaN to 0."""
    whole = positive_codes(code)
    a = torch.nan_to_num(y.abs(), nan=0.0).clamp(max=float(whole[-1]))
    above = torch.searchsorted(whole, a.contiguous()).clamp(max=len(whole) - 1)
    below = (above - 1).clamp(min=0)
    up, down = whole[above] - a, a - whole[below]
    take = (up < down) | ((up == down) & (above % 2 == 0))
    return torch.copysign(torch.where(take, whole[above], whole[below]), torch.nan_to_num(y, nan=0.0)) + 0.0


def append(k, v, k_scale, v_scale, K, V, slots, d, block, code):
    """The cache's code values (float64, k [N][h][block][row], v [N][h][row][block]) and scales (fp32) after an append."""
    out = []
    runs = {}
    for t, s in enumerate(slots):
        if 0 <= s < k.shape[0] * block:
            runs.setdefault(s // block, []).append((s % block, t))
    for codes, scale, x in ((k.clone(), k_scale.clone(), K), (v.transpose(2, 3).clone(), v_scale.clone(), V)):
        x = x.detach().cpu().double()
        for b, rows in runs.items():
            for h in range(x.shape[1]):
                new = x[[t for _, t in rows], h]
                size = torch.where(torch.isfinite(new), new.abs(), torch.zeros_like(new))
                s0 = torch.zeros(()) if any(o == 0 for o, _ in rows) else scale[b, h].clone()
                s1 = torch.maximum(s0, (size.max().float() / torch.tensor(MOST[code])))
                if float(s0) == 0.0 and any(o == 0 for o, _ in rows):
                    codes[b, h] = 0.0
                elif s1 > s0:
                    codes[b, h] = nearest(codes[b, h] * s0.double() / s1.double(), code)
                for o, t in rows:
                    y = x[t, h] / s1.double() if float(s1) > 0 else torch.zeros_like(x[t, h])
                    codes[b, h, o, :d] = nearest(y, code)
                scale[b, h] = s1
        out += [codes, scale]
    return out[0], out[2].transpose(2, 3), out[1], out[3]


def cache_map(lengths, news, table, free, block, n_slots):
    table = [list(r) for r in table]
    width = len(table[0]) if table else 0
    starts, slots, used = [0], [], 0
    for i, (length, new) in enumerate(zip(lengths, news)):
        length = min(max(length, 0), width * block)
        new = min(max(new, 0), length)
        before = length - new
        for b in range(-(-before // block), -(-length // block)):
            table[i][b] = free[used] if used < len(free) else -1
            used += 1
        for j in range(before, length):
            b = table[i][j // block]
            slots.append(b * block + j % block if b >= 0 else -1)
        starts.append(starts[-1] + new)
    slots = (slots + [-1] * n_slots)[:n_slots]
    return table, starts, slots, used


def cache_attention(Q, k, v, k_scale, v_scale, table, lengths, d, block, scale=None, cap=0.0, slopes=None):
    """(O, bound) in float64 [batch][nq][hq][d] from code values (float64) and scales."""
    eps = torch.finfo(Q.dtype).eps / 2
    tiny = 2.0 ** -25 if Q.dtype == torch.float16 else 2.0 ** -134
    Q = Q.detach().double().cpu()
    batch, nq, hq, _ = Q.shape
    hkv = k.shape[1]
    scale = d ** -0.5 if scale is None else scale
    O, most = torch.zeros_like(Q), torch.zeros_like(Q)
    for b in range(batch):
        length = min(max(lengths[b], 0), len(table[b]) * block)
        js = [j for j in range(length) if 0 <= table[b][j // block] < k.shape[0]]
        if not js:
            most[b] += tiny
            continue
        at = torch.tensor([table[b][j // block] for j in js])
        off = torch.tensor([j % block for j in js])
        j = torch.tensor(js)
        p = torch.arange(length - nq, length)[:, None]
        seen = j[None, :] <= p
        for h in range(hq):
            f = h * hkv // hq
            kk = k[at, f, off, :d] * k_scale[at, f].double()[:, None]
            vc, vs = v[at, f, :d, off], v_scale[at, f].double()
            vv = vc * vs[:, None]
            q = Q[b, :, h]
            u = scale * q @ kk.T
            err = STEP32 * (d + 12) * scale * q.abs() @ kk.abs().T
            s = cap * torch.tanh(u / cap) if cap else u
            if cap:
                err = err + 16 * STEP32 * cap
            if slopes is not None:
                s = s - float(slopes[h]) * (p - j).abs()
                err = err + 4 * STEP32 * float(slopes[h]) * (p - j).abs()
            err = err + 8 * STEP32 * (1 + s.abs())
            s = s.masked_fill(~seen, -math.inf)
            P = torch.nan_to_num(torch.softmax(s, 1), nan=0.0)
            err = 2 * torch.where(seen, err, torch.zeros_like(err)).amax(1, keepdim=True)
            O[b, :, h] = P @ vv
            # probabilities in f16, a step of 2^-24 at the least, times the largest scale
            most[b, :, h] = 1.01 * ((2.0 ** -11 + 2 * err + 4 * STEP32) * (P @ vv.abs()) +
                                    2.0 ** -25 * float(vs.max()) * (seen.double() @ vc.abs()) + eps * O[b, :, h].abs() + tiny)
    return O, most
