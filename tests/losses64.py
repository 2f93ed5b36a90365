"""The losses on rows of logits in 64 bits on the CPU, with their gradients by formula, and how far the library's fp32 may be from
them.  Not collected by pytest.

Bounds, in units of u = 2^-24 (half a step of fp32).  A term exp(z - max) of a row's sum: z - max is rounded once (u |z - max|), times
log2 e twice (the constant, the product), the instruction is off by 2 u: u (3 |z - max| + 2) of the term.  Over the sum that is
u (3 E + 2) with E the mean of |z - max| under the row's probabilities (a rescale's exponent is a part of the same distance, so it adds
nothing to E).  Beside that a rescale and an addition are four roundings: a thread's chain is 16 numbers a step, then a rescale a
step, then at most 6 joins over lanes, 16 over wavefronts and one a piece.  So the sum, and with it log p, is off by
  delta = u (3 E + 2 + adds),  adds = 16 + 4 steps + 4 (22 + pieces),  steps and pieces <= ceil(n / 4096);
what follows is in 64 bits and rounded once at the end."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
STEP = {"float32": U, "bfloat16": 2.0 ** -8}          # half a step of the outputs' types, relative


def rows64(z, tokens, ids=None, weight=None, inside=None):
    """per row: z float64 array of live columns.  Returns dicts with lp, p, col, delta; None for a row that does not count"""
    out = []
    for r, x in enumerate(z):
        if (weight is not None and weight[r] == 0) or (inside is not None and not inside[r]):
            out.append(None)
            continue
        x = np.asarray(x, np.float64)
        n, t = len(x), int(tokens[r])
        if ids is None:
            col = t if 0 <= t < n else -1
        else:
            at = np.searchsorted(ids[r], t)
            col = int(at) if at < n and ids[r][at] == t else -1
        with np.errstate(all="ignore"):
            top = x.max(initial=-np.inf)
            gap = np.where(x == -np.inf, -np.inf, x - (top if np.isfinite(top) else 0.0)) if not np.isnan(x).any() else x * np.nan
            e = np.exp(gap)
            s = e.sum()
            if np.isposinf(top):
                s = np.nan
            p = e / s if s != 0 else e
            lp = -np.inf if col < 0 or x[col] == -np.inf else gap[col] - np.log(s)
            mean = float(np.nansum(np.where(p > 0, p * -gap, 0.0))) if np.isfinite(s) else 0.0
        pieces = -(-max(n, 1) // 4096)
        delta = U * (3 * mean + 2 + 16 + 4 * pieces + 4 * (22 + pieces))
        out.append(dict(lp=lp, p=p, gap=gap, col=col, delta=delta, has=not lp < -745.0))
    return out


def gradient(rows, widths, dlp, slack, scale=1.0, kind="float32"):
    """[(gradient, bound)] of rows whose loss changes by dlp[r] with log p; slack[r]: how far dlp itself may be off"""
    out = []
    for q, n, c, off in zip(rows, widths, dlp, slack):
        if q is None or not q["has"]:
            out.append((np.zeros(n), np.zeros(n)))
            continue
        with np.errstate(all="ignore"):
            c, off = c * scale, off * abs(scale)
            g = -c * q["p"]
            g[q["col"]] += c
            here = np.zeros(n)
            here[q["col"]] = 1.0
            gap = np.where(np.isfinite(q["gap"]), np.abs(q["gap"]), 0.0)
            # p: the exponent as above, the sum's error, c / sum and the product rounded; the token's entry: c rounded, the sum rounded
            bound = off * (here + q["p"]) + abs(c) * q["p"] * (U * (3 * gap + 6) + q["delta"]) + here * 2 * U * abs(c) + 2.0 ** -140
            bound = bound + STEP[kind] * (np.abs(g) + bound)
            # exp2 of the instruction is 0 where the result is a denormal
            bound = bound + abs(c) * 2.0 ** -125
        out.append((g, bound))
    return out


def policy(rows, old, ref, adv, weight, lo, hi, beta):
    """(loss, its bound, row losses, their bounds, dlp, slack of dlp).  A ratio nearer to a border than it may be off -- delta of itself -- may
    fall on either side: the loss is continuous there, its derivative is -ratio A on one side and 0 on the other"""
    R = len(rows)
    row, bound, dlp, slack = np.zeros(R), np.zeros(R), np.zeros(R), np.zeros(R)
    total = terms = 0.0
    lo, hi, beta = float(np.float32(lo)), float(np.float32(hi)), float(np.float32(beta))
    with np.errstate(all="ignore"):
        for r, q in enumerate(rows):
            if q is None or not q["has"]:
                continue
            w = 1.0 if weight is None else float(weight[r])
            a, ratio = float(adv[r]), np.exp(q["lp"] - float(old[r]))
            free, held = ratio * a, float(np.clip(ratio, 1 - lo, 1 + hi)) * a
            x = -min(free, held) if free == free else free
            c = -free if free <= held or free != free else 0.0
            off, coff = abs(free) * q["delta"], abs(c) * q["delta"]
            if min(abs(ratio - (1 - lo)), abs(ratio - (1 + hi))) <= 1.01 * q["delta"] * ratio:
                coff = 1.01 * abs(free)
            if beta != 0:
                gap = float(ref[r]) - q["lp"]
                e = np.exp(gap)
                x += beta * (e - gap - 1)
                c += beta * (1 - e)
                off += abs(beta) * abs(1 - e) * q["delta"] + abs(beta) * e * q["delta"] ** 2
                coff += abs(beta) * e * q["delta"]
            row[r], bound[r] = x, 1.001 * off + U * (abs(x) + off) + 1e-15 * (1 + abs(x))
            dlp[r], slack[r] = w * c, abs(w) * (1.001 * coff + 1e-15)
            total += w * x
            terms += abs(w) * bound[r]
    return total, terms + U * (abs(total) + terms) + 1e-300, row, bound, dlp, slack


def preference(rows, off, ref, weight, beta, smoothing):
    """(loss, its bound, margins, their bounds, dlp, slack of dlp)"""
    R, pairs = len(rows), (len(off) - 1) // 2
    beta, smoothing = float(np.float32(beta)), float(np.float32(smoothing))
    dlp, slack = np.zeros(R), np.zeros(R)
    margin, mb, loss, lb = np.zeros(pairs), np.zeros(pairs), 0.0, 0.0
    w_of = lambda r: 1.0 if weight is None else float(weight[r])
    for p in range(pairs):
        s = d = 0.0
        for sign, q in ((1, 2 * p), (-1, 2 * p + 1)):
            for r in range(off[q], off[q + 1]):
                if rows[r] is not None and rows[r]["has"]:
                    s += sign * w_of(r) * (rows[r]["lp"] - (0.0 if ref is None else float(ref[r])))
                    d += abs(w_of(r)) * rows[r]["delta"]
        with np.errstate(all="ignore"):
            m = beta * s
            dm = 1.001 * abs(beta) * d
            margin[p], mb[p] = m, dm + U * (abs(m) + dm)
            loss += ((1 - smoothing) * np.logaddexp(0, -m) + smoothing * np.logaddexp(0, m)) / pairs
            lb += dm / pairs
            slope = -(1 - smoothing) / (1 + np.exp(m)) + smoothing / (1 + np.exp(-m))
            for sign, q in ((1, 2 * p), (-1, 2 * p + 1)):
                for r in range(off[q], off[q + 1]):
                    dlp[r] = sign * beta / pairs * w_of(r) * slope
                    slack[r] = abs(beta) / pairs * abs(w_of(r)) * (0.2501 * dm + 1e-14)
    return loss, 1.001 * lb + U * (abs(loss) + lb) + 1e-15, margin, mb + 1e-15, dlp, slack
