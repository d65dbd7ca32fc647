"""Attention and its gradient from their formulas in 64 bits, entry by entry, for inputs that attn_formulas.py does
not allow for: entries that are not finite, caps and magnitudes over the whole accepted range.  Test infrastructure only.

Bounds, u = eps / 2 of the type:
  a score     32-bit product of d terms; a cap adds 16 steps of 2^-24 of the cap where it is 64 or less, else of the
              score itself (the kernels have two forms of tanh); slopes and the exponential a few steps of what they act on
  a weight    rounded once to the type, f16 with its powers of two moved up: by 2^7 and more above the largest one,
              so that half of the smallest step, 2^-25, is 2^-32 of it; in dV by 2^14: 2^-39
  ds          rounded once to the type, f16 times a power of two that puts the largest |<dO, V> - <dO, O>| of some of what is seen at 2^8
              (dK: 2^4) or more, or the largest |ds| at 2^14: half of the smallest step is 2^-33 (2^-29) of the largest that is seen
"""
import math

import torch

STEP32 = 2.0 ** -24


def _masked(weights, seen, x):
    """sum_j weights_ij x_j over the seen j alone: what is not finite elsewhere does not meet a zero."""
    out = torch.zeros(weights.shape[0], x.shape[1], dtype=torch.float64)
    plain = torch.isfinite(x).all(1)
    out += torch.where(seen, weights, torch.zeros_like(weights))[:, plain] @ x[plain]
    for j in (~plain).nonzero().flatten().tolist():
        out += torch.where(seen[:, j:j + 1], weights[:, j:j + 1] * x[j:j + 1], torch.zeros(()).double())
    return out


def attention(Q, K, V, dO=None, scale=None, causal=False, cap=0.0, slopes=None, starts=None, k_starts=None, prefix=None):
    """As attn_formulas.attention: O, lse, dQ, dK, dV and their bounds under name + "+".  Entries that have to be
    not finite are NaN in the value and infinite in the bound; rows and keys outside the documents NaN with a bound of 0."""
    f16 = Q.dtype == torch.float16
    eps = torch.finfo(Q.dtype).eps / 2
    tiny = 2.0 ** -25 if f16 else 2.0 ** -134
    small_P, small_dV, small_ds = (2.0 ** -32, 2.0 ** -39, 2.0 ** -33) if f16 else (2.0 ** -134, 2.0 ** -134, 0.0)
    Q, K, V = (t.detach().double().cpu() for t in (Q, K, V))
    dO = None if dO is None else dO.detach().double().cpu()
    (n, hq, d), (m, hkv, _) = Q.shape, K.shape
    scale = d ** -0.5 if scale is None else scale
    if starts is None:
        starts, k_starts = [0, n], [0, m]
    elif k_starts is None:
        k_starts = starts
    nan = float("nan")
    r = {"O": torch.full((n, hq, d), nan).double(), "lse": torch.full((hq, n), nan).double()}
    for name, like in (("dQ", Q), ("dK", K), ("dV", V)):
        r[name] = torch.full_like(like, nan)
    for name in list(r):
        r[name + "+"] = torch.zeros_like(r[name])
    group = hq // hkv
    for c in range(len(starts) - 1):
        q0, q1, k0, k1 = starts[c], starts[c + 1], k_starts[c], k_starts[c + 1]
        nq, nk = q1 - q0, k1 - k0
        p, j = torch.arange(nq)[:, None] + nk - nq, torch.arange(nk)[None, :]
        visible = ((j <= p) | (j < (0 if prefix is None else prefix[c]))) if causal else torch.ones(nq, nk, dtype=torch.bool)
        for f in range(hkv):
            k, v = K[k0:k1, f], V[k0:k1, f]
            all_ds, all_off, all_q, all_seen = [], [], [], []
            for name in ("dK", "dV"):
                r[name][k0:k1, f] = 0.0
            by_key = torch.zeros(nk, 1, dtype=torch.float64)  # |<dO, V> - <dO, O>| of who sees a key, at most
            for h in range(f * group, (f + 1) * group):
                q = Q[q0:q1, h]
                finite_k, finite_q = torch.nan_to_num(k, 0, 0, 0).abs(), torch.nan_to_num(q, 0, 0, 0).abs()
                size = scale * (finite_q @ finite_k.T)
                u = scale * (q @ k.T)
                off = STEP32 * (d + 8) * size
                s, steep = u, torch.ones_like(u)
                if cap:
                    t = torch.tanh(u / cap)
                    s, steep = cap * t, 1 - t * t
                    off = off + 16 * STEP32 * (cap if cap <= 64 else torch.nan_to_num(s, 0, 0, 0).abs())
                if slopes is not None:
                    far = float(slopes[h]) * (p - j).abs().double()
                    s = s - far
                    off = off + 4 * STEP32 * far
                off = off + 8 * STEP32 * (1 + torch.nan_to_num(s, 0, 0, 0).abs())
                s = s.masked_fill(~visible, -math.inf)
                seen = visible & ~(s == -math.inf).all(1, keepdim=True)  # all scores -infinity: sees no key
                some = seen.any(1)
                top = s.amax(1, keepdim=True) if nk else torch.full((nq, 1), -math.inf).double()
                lse = torch.logsumexp(s, 1) if nk else top[:, 0]
                lse = torch.where(top[:, 0] == math.inf, torch.full_like(lse, nan), lse)
                P = torch.where(seen, torch.exp(s - lse[:, None]), torch.zeros_like(s))
                err = 2 * torch.where(seen, off, torch.zeros_like(off)).amax(1, keepdim=True) if nk else torch.zeros(nq, 1).double()
                O = _masked(P, seen, v)
                # an entry of V that is not finite reaches who sees it, however small its weight
                for x in (~torch.isfinite(v).all(1)).nonzero().flatten().tolist():
                    who = (seen[:, x] & (s[:, x] > -math.inf))[:, None]
                    O = torch.where(who & ~torch.isfinite(v[x])[None], O + torch.where(torch.isfinite(v[x]), 0.0, v[x]), O)
                    O = torch.where(torch.isnan(lse)[:, None], torch.full_like(O, nan), O)
                size_v = torch.nan_to_num(v, 0, 0, 0).abs()
                offO = (eps + 2 * err) * (torch.nan_to_num(P, 0) @ size_v) + small_P * (seen.double() @ size_v) + \
                    eps * torch.nan_to_num(O, 0, 0, 0).abs() + tiny
                r["O"][q0:q1, h], r["lse"][h, q0:q1] = O, lse
                r["O+"][q0:q1, h] = torch.where(torch.isnan(O), math.inf, 1.01 * offO)
                r["lse+"][h, q0:q1] = torch.where(torch.isnan(lse), math.inf, err[:, 0] + 8 * STEP32 * torch.where(
                    some, torch.nan_to_num(lse, 0, 0, 0).abs(), torch.zeros_like(lse)))
                if dO is None:
                    continue
                g = dO[q0:q1, h]
                # rows with an entry of Q, dO or O that is not finite: NaN in their dQ and in dK, dV of what they see
                bad = some & ~(torch.isfinite(q) & torch.isfinite(g) & torch.isfinite(O)).all(1)
                P = torch.where(seen & bad[:, None], nan, P)
                g0 = torch.where(some[:, None], g, torch.zeros_like(g))
                D = (g0 * torch.where(some[:, None], O, torch.zeros_like(O))).sum(1, keepdim=True)
                raw = g0 @ v.T - D
                ds = torch.where(seen, P * raw * steep, torch.zeros_like(P))
                size_g = torch.nan_to_num(g0, 0, 0, 0).abs()
                off_in = STEP32 * (d + 4) * (size_g @ size_v.T + (size_g * torch.nan_to_num(O, 0, 0, 0).abs()).sum(1, keepdim=True)) + \
                    (size_g * offO).sum(1, keepdim=True)
                fine = torch.nan_to_num(ds, 0, 0, 0).abs()
                off_ds = (eps + err + 8 * STEP32) * fine + torch.nan_to_num(P * off_in * steep, 0, 0, 0) + tiny * 2.0 ** -24
                if cap:
                    off_ds = off_ds + torch.nan_to_num(P * raw.abs(), 0, 0, 0) * (2 * off / cap + 16 * STEP32)
                off_ds = torch.where(seen, off_ds, torch.zeros_like(off_ds))
                all_ds.append(ds), all_off.append(off_ds), all_q.append(q), all_seen.append(seen)
                met = torch.where(seen, torch.nan_to_num(g0 @ v.T, 0, 0, 0).abs(), torch.zeros_like(P))
                most = 2 * met.amax(1, keepdim=True) if nk else torch.zeros(nq, 1).double()  # (O is a mean of V)
                if nq and nk:
                    by_key = torch.maximum(by_key, torch.where(seen, met + most / 2, torch.zeros_like(met)).amax(0)[:, None])
                dQ = scale * _masked(ds, seen, k)
                # one of K that is not finite: NaN in dQ of the rows that see it
                meets = (seen & ~torch.isfinite(k).all(1)[None]).any(1)
                dQ = torch.where(meets[:, None], nan, dQ)
                off = scale * ((off_ds + (nk + 4) * STEP32 * fine) @ finite_k + small_ds * most * (seen.double() @ finite_k))
                r["dQ"][q0:q1, h] = dQ
                r["dQ+"][q0:q1, h] = torch.where(torch.isnan(dQ), math.inf, 1.01 * (off + eps * dQ.abs() + tiny))
                off_P = torch.where(seen, (eps + err) * torch.nan_to_num(P, 0) + small_dV, torch.zeros_like(P))
                r["dV"][k0:k1, f] += _masked(P.T, seen.T, g)
                r["dV+"][k0:k1, f] += 1.01 * ((off_P + (nq * hq + 4) * STEP32 * torch.nan_to_num(P, 0)).T @ size_g)
            if dO is None or not nq or not nk:
                continue
            for ds, off_ds, q, seen in zip(all_ds, all_off, all_q, all_seen):
                size_q = torch.nan_to_num(q, 0, 0, 0).abs()
                r["dK"][k0:k1, f] += scale * _masked(ds.T, seen.T, q)
                r["dK+"][k0:k1, f] += 1.01 * scale * ((off_ds + (nq * hq + 4) * STEP32 * torch.nan_to_num(ds, 0, 0, 0).abs()).T @ size_q +
                                                      16 * small_ds * by_key * (seen.double().T @ size_q))
    for c in range(len(starts) - 1):  # a gradient that is not finite: whichever way
        for name, at in (("dQ", slice(starts[c], starts[c + 1])), ("dK", slice(k_starts[c], k_starts[c + 1])),
                         ("dV", slice(k_starts[c], k_starts[c + 1]))):
            x = r[name][at]
            if name != "dQ":
                r[name + "+"][at] += eps * x.abs() + tiny
            r[name + "+"][at][~torch.isfinite(x)] = math.inf
            x[~torch.isfinite(x)] = nan
    return r


def compare(name, got, r):
    """got against r[name]: within the bound, the same infinity, or not finite where the value is NaN with an infinite bound."""
    got, want, most = got.double().cpu(), r[name], r[name + "+"]
    outside = torch.isnan(want) & (most == 0)
    lost = torch.isnan(want) & (most == math.inf)
    same = torch.where(torch.isinf(want), got == want, (got - want).abs() <= most)
    same = torch.where(lost, ~torch.isfinite(got), same) | outside
    if not same.all():
        at = (~same).nonzero()[0].tolist()
        raise AssertionError(f"{name}: {int((~same).sum())} of {int((~outside).sum())} off, first at {at}: got {float(got[tuple(at)])}, "
                             f"want {float(want[tuple(at)])} within {float(most[tuple(at)])}")
    fine = torch.isfinite(want) & torch.isfinite(most)
    return float(((got - want).abs()[fine] / most[fine].clamp(min=1e-300)).max()) if fine.any() else 0.0
