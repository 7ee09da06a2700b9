"""Attention over a paged VQ cache in 64 bits, all rows of a head at once, for the tests of vq_attn_paged (test_paged.Case gives the inputs)."""
import numpy as np

U = 2.0 ** -24     # half a step of fp32, relative


def attend(case):
    """(out, bound on the error of an fp32 computation with fp16 weights) [rows][Hq][D].

    Bound, term by term: a score is a sum of D exact products in fp32 in some order, D + 2 roundings of sum |q k|, scaled.  A capped one
    is cap (1 - 2 / (2^x + 1)), in units of cap U: its factors' rounding 2 + 2, 2^x 1, the sum 2, the reciprocal 4, product and difference 3: 14, for a cap of 256
    2^-12, half of what a weight's rounding allows.  Under a larger cap that form serves only where |x| = |2 log2(e) s / cap| passes 1 in a row, the cap then being
    below 2.9 times the row's largest score, so that the error never grows with the cap; elsewhere an odd polynomial of the score, 6 roundings of the
    result.  A biased score: 4 roundings of the bias.  2^x and the difference to the
    maximum: 4 of the score and of the largest.  A weight is rounded to a half (2^-11 of it, 2^-31 of the largest where it is a subnormal one; below
    that it may vanish); the output is (2^-11)."""
    Hq = case.H * case.group
    out, bound = np.zeros((case.rows, Hq, case.D)), np.zeros((case.rows, Hq, case.D))
    for b, (ln, n) in enumerate(case.reqs):
        if n == 0 or ln == 0:
            continue
        K, V = case.values(case.K_codes[b], case.k_cb), case.values(case.V_codes[b], case.v_cb)
        t, pos = np.arange(ln)[None], (ln - n + np.arange(n))[:, None]
        see = t <= pos
        if case.window:
            see &= t > pos - case.window
        if case.prefix is not None:
            see |= t < case.prefix[b]
        some = see.any(1)
        rows = slice(case.cu[b], case.cu[b] + n)
        for hq in range(Hq):
            k, val, q = K[:, hq // case.group], V[:, hq // case.group], case.q[rows, hq].astype(np.float64)
            s = case.sm_scale * (q @ k.T)
            ds = abs(case.sm_scale) * (case.D + 2) * U * (np.abs(q) @ np.abs(k).T)
            if case.softcap:
                top = np.where(see, np.abs(s), 0.0).max(1, keepdims=True)
                s = case.softcap * np.tanh(s / case.softcap)
                ds = ds + 6 * U * np.abs(s) + 14 * U * (case.softcap if case.softcap <= 256 else np.where(
                    2.885 * top < 0.999 * case.softcap, 0.0, np.minimum(case.softcap, 2.9 * top)))
            if case.slopes is not None:
                bias = float(case.slopes[hq]) * np.abs(pos - t)
                s = s - bias
                ds = ds + 4 * U * np.abs(bias)
            ds = ds + 4 * U * (np.abs(s) + np.where(see, np.abs(s), 0.0).max(1, keepdims=True))
            s = np.where(see, s, -np.inf)
            m = np.where(some, s.max(1), 0.0)[:, None]
            p = np.exp(s - m)
            p /= np.where(some, p.sum(1), 1.0)[:, None]
            pe = p * (2.0 ** -11 + np.expm1(np.where(see, ds, 0.0)))
            o = p @ val
            out[rows, hq] = o
            bound[rows, hq] = (2.0 ** -11 * np.abs(o) + pe @ np.abs(val) + pe.sum(1)[:, None] * np.abs(o)
                               + see.sum(1)[:, None] * 2.0 ** -31 * np.abs(val).max() + some[:, None] * 2.0 ** -25)
    return out, bound * 1.01      # (products of the small terms)


def check(case, got):
    want, bound = attend(case)
    got = got.float().cpu().numpy().astype(np.float64)[:case.rows]
    assert np.isfinite(got).all()
    worst = np.abs(got - want) / np.maximum(bound, 1e-30)
    at = np.unravel_index(np.argmax(worst), worst.shape) if worst.size else None
    assert worst.size == 0 or worst[at] <= 1.0, (at, worst[at], got[at], want[at])
