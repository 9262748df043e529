"""The cache operators in 64 bits, from their definitions (numpy, CPU), and the error bounds of their tests."""
import numpy as np

D = 128


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def attention(q, k, v, n, n_init, n_local, scale=None, pk=None, pv=None):
    """One sequence.  q [Hq, T, D], k, v [Hkv, cap, D], n tokens; pk, pv [Hkv, P, D]: a prefix that every row sees.

    Returns o [Hq, T, D], w [Hkv, n] (column sums over a group's rows, own keys only), and for the bounds
    mag [Hq, T, D] = sum_j p_ij |v_j| and slack [Hq, T] = bound of the relative error of a p_ij.

    Slots that a row does not see are not touched, so what they hold does not matter.
    slack: logits are sums of 128 fp32 products (exact products of bf16), off by at most 128 * 2^-24 of the sum of
    their magnitudes however they are ordered, plus three roundings of the scaled logit; each enters p through
    its own and the largest logit, so twice.  The row sum adds one rounding per key, the exponentials and the
    division some units of 2^-23.
    """
    hq, T, _ = q.shape
    hkv = k.shape[0]
    group = hq // hkv
    c = 1.0 / np.sqrt(D) if not scale else scale
    o, mag, slack, w = np.zeros(q.shape), np.zeros(q.shape), np.zeros((hq, T)), np.zeros((hkv, n))
    for h in range(hq):
        kv = h // group
        for t in range(T):
            i = n - T + t
            if i < 0:
                continue
            j = np.arange(i + 1)
            j = j[(j < n_init) | (i - j < n_local)]
            keys, vals = k[kv, j], v[kv, j]
            if pk is not None:
                keys, vals = np.concatenate([pk[kv], keys]), np.concatenate([pv[kv], vals])
            s = (keys @ q[h, t]) * c
            p = np.exp(s - s.max())
            p /= p.sum()
            o[h, t] = p @ vals
            mag[h, t] = p @ np.abs(vals)
            w[kv, j] += p[len(p) - len(j):]
            terms = (np.abs(keys) @ np.abs(q[h, t])).max() * c
            slack[h, t] = 2 * (128 + 3) * 2.0 ** -24 * terms + (len(p) + 16) * 2.0 ** -23
    return o, w, mag, slack


P_TWO_BF16 = 2.0 ** -16    # P as the sum of two bf16: what is left of p after one half step is rounded again
P_BF16 = 2.0 ** -8         # P as one bf16 (more than 32 rows of a K/V head): off by half a step, 2^-8 of the value


def check_o(got, want, mag, slack, what="", p_step=P_TWO_BF16):
    """bf16 output: half a step of the value (2^-8); every p_ij that multiplies v_j is off by p_step of itself, which
    moves the output by at most p_step * sum_j p_ij |v_j|; the p's own error in the same way."""
    got = f64(got)
    assert np.isfinite(got).all(), f"{what}: not finite"
    bound = 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * (p_step + slack[..., None]) * mag + 1e-30
    over = np.abs(got - want) / bound
    assert over.max(initial=0.0) <= 1.0, f"{what}: error {over.max():.3g} times its bound at {np.unravel_index(over.argmax(), over.shape)}"


def check_w(got, want, slack, what=""):
    """fp32 sums of p: the p's own error, and one rounding per row."""
    got = f64(got)
    bound = want * (slack.max(initial=0.0) + slack.size * 2.0 ** -24) + 1e-30
    over = np.abs(got - want) / bound
    assert over.max(initial=0.0) <= 1.0, f"{what}: error {over.max():.3g} times its bound at {np.unravel_index(over.argmax(), over.shape)}"


def evict(weight, n, n_init, n_recent, keep):
    """Kept slots, ascending, of one sequence and K/V head (weight [n] float)."""
    if n <= keep:
        return np.arange(n)
    w = np.asarray(weight[:n], dtype=np.float64)
    middle = list(range(n_init, n - n_recent))
    # largest first; NaN behind everything; ties: lower slot
    middle.sort(key=lambda j: (1, 0.0, j) if np.isnan(w[j]) else (0, -w[j], j))
    chosen = middle[:keep - n_init - n_recent]
    return np.array(sorted(list(range(n_init)) + chosen + list(range(n - n_recent, n))), dtype=np.int64)
