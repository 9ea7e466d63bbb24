"""Float64 CPU oracle of the operators around the loss pass (test infrastructure only): 4-bit blocks and their product,
verification of drafted tokens, gradient norm and clipping.  Written from the definitions in include/fopd.h; shares no code
with the library."""

import math

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_blocks(x):
    """(codes [R, d] 0..15, exponents [R, ceil(d / 32)]: 255 for a block of NaN, values [R, d]) of a float array."""
    x = np.asarray(x, dtype=np.float64)
    R, d = x.shape
    nb = (d + 31) // 32
    codes, exps, values = np.zeros((R, d), np.int64), np.zeros((R, nb), np.int64), np.zeros((R, d))
    for b in range(nb):
        blk = x[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(blk).all(axis=1)
        top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(blk), blk, 0.0)).max(axis=1))
        e = np.frexp(top)[1] - 1                            # top = m 2^e, 1 <= m < 2
        s = np.where(top > 0, np.maximum(e - 2, -127), -127)
        unit = np.ldexp(1.0, s)[:, None]
        a = np.minimum(np.abs(np.where(bad[:, None], 0.0, np.where(np.isfinite(blk), blk, 0.0))) / unit, 6.0)
        dist = np.abs(a[:, :, None] - GRID)
        near = dist == dist.min(axis=2, keepdims=True)      # one, or two neighbours at a tie: the even code
        even = near & (np.arange(8) % 2 == 0)
        pick = np.where(near.sum(axis=2) == 2, even.argmax(axis=2), near.argmax(axis=2))
        c = np.where(bad[:, None], 0, pick + 8 * np.signbit(np.where(np.isfinite(blk), blk, 0.0)))
        codes[:, 32 * b:32 * b + 32] = c
        exps[:, b] = np.where(bad, 255, s + 127)
        v = np.where(np.signbit(blk), -GRID[pick], GRID[pick]) * unit
        values[:, 32 * b:32 * b + 32] = np.where(bad[:, None], np.nan, v)
    return codes, exps, values


def mx4_packed(x):
    """The packed matrix byte by byte, as the header describes it."""
    codes, exps, _ = mx4_blocks(x)
    R, d = codes.shape
    steps, groups = (d + 255) // 256, (R + 63) // 64
    out = np.zeros(groups * steps * 8704, np.uint8)
    for row in range(R):
        for col in range(d):
            r, k = row % 64, col % 256
            base = ((row // 64) * steps + col // 256) * 8704
            out[base + (r // 16 * 2 + k // 128) * 1024 + (16 * (k // 32 % 4) + r % 16) * 16 + k % 32 // 2] |= codes[row, col] << (4 * (k % 2))
            out[base + 8192 + 8 * (16 * (k // 32 % 4) + r % 16) + 2 * (r // 16) + k // 128] = exps[row, col // 32]
    return out


def verify(target, draft, draft_ids, first_rows, lens, taus, u, noise):
    """Per sample: kept, token (None: no distribution), log-probs of the tokens 0 .. kept, and margin: how far the nearest
    decision is from turning, as a relative distance (a greedy sample has none).  draft: [R, V], or None for drafts that were looked up; taus[i] = 0 or
    noise None: greedy."""
    out = []
    for i, n in enumerate(lens):
        tau = 0.0 if noise is None else float(taus[i])
        logps, margin, kept = [], math.inf, 0
        while True:
            r = int(first_rows[i]) + kept
            z = np.asarray(target[r], np.float64)
            ok = not np.isnan(z).any() and z.max() > -math.inf and z.max() < math.inf
            if not ok:
                out.append(dict(kept=kept, token=None, logps=logps, margin=margin))
                break
            s = (z - z.max()) / (tau if tau > 0 else 1.0)
            with np.errstate(divide="ignore"):
                lp = s - math.log(np.exp(s).sum())
            p = np.exp(lp)
            q = np.zeros_like(p)
            x = int(draft_ids[r]) if kept < n else -1
            inside = 0 <= x < p.size
            if kept < n and tau > 0:
                if draft is None:
                    if inside:
                        q[x] = 1.0
                else:
                    zq = np.asarray(draft[r], np.float64)
                    if np.isnan(zq).any() or not -math.inf < zq.max() < math.inf:
                        out.append(dict(kept=kept, token=None, logps=logps, margin=margin))
                        break
                    sq = (zq - zq.max()) / tau
                    q = np.exp(sq) / np.exp(sq).sum()
            if kept < n and inside:
                if tau == 0:
                    keep = x == int(np.argmax(z))
                else:
                    uq = float(u[r]) * q[x]
                    keep = uq < p[x]
                    margin = min(margin, abs(uq - p[x]) / max(uq, p[x]) if max(uq, p[x]) > 0 else math.inf)
                if keep:
                    logps.append(float(lp[x]))
                    kept += 1
                    continue
            if tau == 0:
                token = int(np.argmax(z))
            else:
                left = np.maximum(p - q, 0.0)
                # (an entry's relative error is that of p and q over their difference)
                sure = np.where(left > 0, left / np.maximum(p + q, 1e-300), 1.0)
                if not left.max() > 0:
                    left, sure = p, np.ones_like(p)
                score = left / np.asarray(noise[i][:p.size], np.float64)
                token = int(np.argmax(score))
                rest = np.delete(score, token)
                second = np.argmax(rest) if rest.size else None
                if rest.size and rest[second] > 0:
                    gap = 1.0 - rest[second] / score[token]
                    margin = min(margin, gap * min(sure[token], np.delete(sure, token)[second]))
            logps.append(float(lp[token]))
            out.append(dict(kept=kept, token=token, logps=logps, margin=margin))
            break
    return out


def verify_logp_tolerance(z, x, tau):
    """How far a 32-bit log-prob may be off: every term exp((z - max) / tau) has an exponent of three roundings (difference, product, log2 e
    / tau), an exponential of one unit in the last place (2^-23) and passes through at most V / 256 + 64 additions; then the rounding
    of the result."""
    z = np.asarray(z, np.float64)
    s = (z - z.max()) / (tau if tau > 0 else 1.0)
    p = np.exp(s) / np.exp(s).sum()
    spread = float((p * np.abs(np.where(p > 0, s, 0.0))).sum()) + abs(float(s[x]))
    lp = abs(float(s[x]) - math.log(np.exp(s).sum()))
    return 2.0 ** -24 * (3.0 * spread + 2.0 + z.size / 256 + 64 + lp)


def grad_clip(grads, max_norm, eps):
    """(sum of squares, norm, coefficient, scaled gradients)."""
    total = math.fsum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads)
    norm = math.sqrt(total)
    c = max_norm / (norm + eps) if norm + eps > 0 else math.inf
    c = 1.0 if c >= 1.0 else c
    return total, norm, c, [np.asarray(g, np.float64) * c for g in grads]
