"""Plain CPU reference of a served verification step -- TEST INFRASTRUCTURE.

Only tests may import this module; it shares no code with the GPU library.  Whole numbers are computed request by request as
the definitions say; attention and verification in float64 from the values that the arrays hold.
"""
import numpy as np


def pages(pages, length, add, table, free, nfree, page, accepted=None, tokens=None):
    """Block tables and slot maps of a step.  Returns a dict of what sd_pages writes; table and free are copies."""
    table, free = np.array(table), np.array(free)
    B, width = table.shape
    tokens = int(np.sum(add)) if tokens is None else tokens
    held = [int(h) for h in pages]
    keep = [min(int(length[b]) + (int(accepted[b]) + 1 if accepted is not None else 0), held[b] * page) for b in range(B)]
    want = [-(-(keep[b] + int(add[b])) // page) for b in range(B)]
    stack = [int(x) for x in free[:nfree]]
    for b in range(B):                                              # surplus pages go back first
        stack += [int(x) for x in table[b, want[b]:held[b]]]
    cu, slot, pos, kv, short = [0], [], [], [], False
    for b in range(B):
        a, served = int(add[b]), want[b] <= width
        if served and want[b] > held[b]:
            short = short or want[b] - held[b] > len(stack)
            served = not short
            if served:
                for i in range(held[b], want[b]):
                    table[b, i] = stack.pop()
        if served:
            held[b] = want[b]
        kv.append(keep[b] + (a if served else 0))
        for i in range(a):
            t = keep[b] + i
            slot.append(int(table[b, t // page]) * page + t % page if served else -1)
            pos.append(t if served else -1)
        cu.append(cu[-1] + a)
    if len(stack) > nfree:
        free[nfree:len(stack)] = stack[nfree:]
    i32 = lambda v: np.array(v, np.int32)  # noqa: E731
    return dict(pages=i32(held), length=i32(keep), kv=i32(kv), nfree=i32([len(stack)]), cu=i32(cu), slot=i32(slot)[:tokens], pos=i32(pos)[:tokens],
                table=table, free=free)


def attend(q, k_cache, v_cache, cu, kv, table, scale, window=0):
    """q [T][Hq][D], caches [pages][page][Hkv][D] -> out, lse and, for error bounds, sum_j w_j |v_j| and the largest
    scale * sum_d |q_d k_jd| of every row, all float64."""
    q = np.asarray(q, np.float64)
    T, Hq, D = q.shape
    page, Hkv = k_cache.shape[1], k_cache.shape[2]
    out, lse, size, big = np.zeros(q.shape), np.full((T, Hq), -np.inf), np.zeros(q.shape), np.zeros((T, Hq))
    for b in range(len(kv)):
        m = int(cu[b + 1]) - int(cu[b])
        j = np.arange(int(kv[b]))
        at = np.asarray(table[b])[j // page] if len(j) else j
        for i in range(m):
            pos = int(kv[b]) - m + i
            lo, hi = max(0, pos - window + 1) if window else 0, pos + 1
            if hi <= lo:
                continue
            k = np.asarray(k_cache[at[lo:hi], j[lo:hi] % page], np.float64)
            v = np.asarray(v_cache[at[lo:hi], j[lo:hi] % page], np.float64)
            for h in range(Hq):
                t, g = int(cu[b]) + i, h // (Hq // Hkv)
                s = scale * (k[:, g] @ q[t, h])
                top = s.max()
                w = np.exp(s - top)
                lse[t, h] = top + np.log(w.sum())
                w /= w.sum()
                out[t, h] = w @ v[:, g]
                size[t, h] = w @ np.abs(v[:, g])
                big[t, h] = scale * (np.abs(k[:, g]) @ np.abs(q[t, h])).max()
    return out, lse, size, big


def _probabilities(rows, tau):
    x = np.array(rows, np.float64)
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, np.finfo(np.float32).max)
    top = x.max(axis=-1, keepdims=True)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(np.isneginf(x), 0.0, np.exp((x - top) / tau))
    total = w.sum(axis=-1, keepdims=True)
    return w / np.where(total == 0, 1.0, total)


def verify_logits(p, q, tok, r, noise, tau, cu):
    """n, next and, per request, how close the nearest decision was (relative): a float32 computation may decide
    otherwise only where that is of its rounding's size."""
    B, V = len(tau), p.shape[1]
    n_out, next_out, close = np.zeros(B, np.int32), np.zeros(B, np.int32), np.full(B, np.inf)
    for b in range(B):
        k, first = int(cu[b + 1]) - int(cu[b]) - 1, int(cu[b]) - b
        rows = np.array(p[cu[b]:cu[b + 1]], np.float64)
        rows[np.isnan(rows)] = -np.inf
        rows = np.minimum(rows, np.finfo(np.float32).max)
        x = np.clip(np.asarray(tok[first:first + k], np.int64), 0, V - 1)
        if not tau[b] > 0:
            best = rows.argmax(axis=1)
            n = next((j for j in range(k) if x[j] != best[j]), k)
            n_out[b], next_out[b] = n, best[n]
            continue
        P = _probabilities(rows, float(tau[b]))
        if q is not None:
            Q = _probabilities(np.asarray(q[first:first + k], np.float64), float(tau[b])) if k else np.zeros((0, V))
        else:
            Q = np.zeros((k, V))
            Q[np.arange(k), x] = 1.0
        n = k
        for j in range(k):
            lhs, rhs = float(r[first + j]) * Q[j, x[j]], P[j, x[j]]
            if max(lhs, rhs) > 0:
                close[b] = min(close[b], abs(lhs - rhs) / max(lhs, rhs))
            if not lhs <= rhs:
                n = j
                break
        w = np.maximum(P[n] - Q[n], 0.0) if n < k else P[n]
        mass = P[n] + Q[n] if n < k else P[n]                       # float32 rounding moves a weight by this much times its unit
        if w.max() == 0:
            w = mass = P[n]
        n_out[b] = n
        if w.max() == 0:
            continue
        with np.errstate(divide="ignore"):
            score = np.where(w > 0, w / np.asarray(noise[b], np.float64), 0.0)
        best = int(score.argmax())
        next_out[b] = best
        if V > 1 and np.isfinite(score[best]):
            with np.errstate(divide="ignore", invalid="ignore"):
                moved = mass / np.asarray(noise[b], np.float64) / score[best]
                gap = (1.0 - score / score[best]) / (moved + moved[best])
            gap[best] = np.inf
            close[b] = min(close[b], float(np.nanmin(gap)))
    return n_out, next_out, close
