"""Infinities, NaN and very large values in slots of V that a row sees, of every kernel of the cache calls: what the
definition in 64 bits gives, sum_j p_ij v_j with p_ij > 0, in the columns that hold such a value and in the others."""
import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests.test_gpu_cache import B, BIG, cache_of, queries, workspace  # noqa: F401  (B: a fixture)

pytestmark = pytest.mark.gpu

# batch, query heads, K/V heads, new tokens, capacity, lengths, n_init, n_local, weights, prefix length (0: none)
CALLS = {
    "workers-1-row": (1, 2, 2, 1, 1500, [1490], 0, BIG, None, 0),
    "workers-window": (1, 8, 2, 1, 1700, [1601], 40, 900, None, 0),
    "workers-weights": (2, 8, 2, 1, 500, [490, 33], 33, 100, "set", 0),
    "workers-4-tokens": (1, 4, 1, 4, 900, [871], 0, BIG, None, 0),
    "workers-two-blocks": (2, 8, 2, 5, 900, [900, 4], 0, BIG, None, 0),
    "one-workgroup": (2, 8, 2, 1, 400, [390, 1], 0, BIG, None, 0),
    "one-workgroup-window": (1, 8, 2, 2, 800, [777], 33, 150, None, 0),
    "shared-20": (1, 20, 1, 1, 2000, [1990], 70, 1000, None, 0),
    "shared-40": (1, 8, 1, 5, 1400, [1390], 0, BIG, "set", 0),
    "shared-132": (1, 4, 1, 33, 1400, [1380], 50, 700, None, 0),
    "shared-many": (75, 16, 4, 20, 200, [199 - i % 7 for i in range(75)], 11, 40, None, 0),
    "prefix-8": (2, 8, 2, 1, 100, [90, 1], 0, BIG, None, 1013),
    "prefix-32": (8, 8, 2, 1, 70, [70, 1, 2, 33, 32, 31, 9, 64], 0, BIG, None, 700),
    "prefix-40": (10, 8, 2, 1, 50, list(range(1, 11)), 0, BIG, None, 1013),
    "prefix-100": (25, 8, 2, 1, 50, list(range(1, 26)), 0, BIG, None, 957),
    "prefix-160": (40, 8, 2, 1, 50, list(range(1, 41)), 0, BIG, None, 1300),
    "prefix-2-tokens": (3, 8, 1, 2, 600, [599, 2, 64], 0, BIG, None, 333),
}


def make(B, case, seed):  # noqa: F811
    batch, hq, hkv, T, cap, lens, n_init, n_local, weights, P = case
    cache = cache_of(B, seed, batch, hkv, cap, lens, weight=weights is not None)
    prefix = cache_of(B, seed + 1, 1, hkv, P + 20, [P], weight=False) if P else None
    return cache, prefix, queries(seed, batch, hq, T)


def run(B, case, cache, prefix, q):  # noqa: F811
    n_init, n_local, weights = case[6:9]
    o = torch.full_like(q, float("nan"))
    if prefix is not None:
        B.minf_prefix_attn(q, o, prefix, cache, workspace(B.minf_prefix_attn_workspace_bytes(q, prefix, cache)))
    else:
        ws = workspace(B.minf_cache_attn_workspace_bytes(q, cache, n_init, n_local, weights))
        B.minf_cache_attn(q, o, cache, ws, n_init=n_init, n_local=n_local, weights=weights)
    torch.cuda.synchronize()
    return o


def wanted(case, cache, prefix, q):
    """Per sequence: n and R.attention's results."""
    hkv, n_init, n_local, P = case[2], case[6], case[7], case[9]
    pk = pv = None
    if P:
        pk, pv = R.f64(prefix.k)[0][:, :P], R.f64(prefix.v)[0][:, :P]
    qd, kd, vd = R.f64(q), R.f64(cache.k), R.f64(cache.v)
    for b, n in enumerate(case[5]):
        yield b, n, R.attention(qd[b], kd[b], vd[b], n, n_init, n_local, None, pk, pv)


def p_step(case):
    rows = case[1] // case[2] * case[3]
    return R.P_BF16 if rows * (case[0] if case[9] else 1) > 64 else R.P_TWO_BF16


def sees(case, n, t, j):
    i = n - case[3] + t
    return i >= 0 and j <= i and (j < case[6] or i - j < case[7])


@pytest.mark.parametrize("name", CALLS)
def test_visible_infinities(B, name):  # noqa: F811
    """Column 2 x + s holds an infinity of sign s in the x-th of some slots, column 20 both signs in two slots, column 21
    NaN in one: the rows that see the slot give it, the others and all other columns what they give without."""
    case = CALLS[name]
    batch, hq, hkv, T, cap, lens, n_init, n_local, weights, P = case
    cache, prefix, q = make(B, case, 60)
    first = lambda n: max(0, n - T - n_local + 1)            # the first slot of the first row's window
    slots = [sorted({0, n // 3, min(first(n), n - 1), n - 1, max(n - T, 0)}) if n else [] for n in lens]
    p_slots = sorted({0, 31, P // 2, P - 2, P - 1}) if P else []
    clean = [wanted(case, cache, prefix, q)]
    special = np.zeros((batch, T, 128), dtype=object)        # 0, "+", "-" or "nan" of each column of a row
    want = list(clean[0])

    def put(v, at, col, value):
        v[..., at, col] = value

    def mark(b, t, col, sign):
        old = special[b, t, col]
        special[b, t, col] = sign if old in (0, sign) else "nan"
    plant = [(1, j, 5 + x) for x, j in enumerate(p_slots)] + [(0, None, x) for x in range(5)]
    for is_prefix, j, x in plant:
        for s, (value, sign) in enumerate(((float("inf"), "+"), (float("-inf"), "-"))):
            col = 2 * x + s
            if is_prefix:
                put(prefix.v, j, col, value)
            for b, n in enumerate(lens):
                if not is_prefix:
                    if x >= len(slots[b]):
                        continue
                    j = slots[b][x]
                    put(cache.v[b], j, col, value)
                for t in range(T):
                    if (n - T + t >= 0) if is_prefix else sees(case, n, t, j):
                        mark(b, t, col, sign)
    for b, n in enumerate(lens):
        if n >= 2:
            for j, value, sign in ((n - 2, float("inf"), "+"), (0, float("-inf"), "-"))[n == 2:]:
                put(cache.v[b], j, 20, value)
                for t in range(T):
                    if sees(case, n, t, j):
                        mark(b, t, 20, sign)
        if n:
            put(cache.v[b], n - 1, 21, float("nan"))
            for t in range(T):
                if sees(case, n, t, n - 1):
                    special[b, t, 21] = "nan"
    o = R.f64(run(B, case, cache, prefix, q))
    for b, n, (ref, w, mag, slack) in want:
        for t in range(T):
            plain = special[b, t] == 0
            for sign, found in (("+", np.isposinf), ("-", np.isneginf), ("nan", np.isnan)):
                cols = np.flatnonzero(special[b, t] == sign)
                assert found(o[b, :, t][:, cols]).all(), f"{name}: sequence {b} token {t} columns {cols} ({sign}): {o[b, :, t][:, cols]}"
            got = torch.from_numpy(o[b, :, t][:, plain])
            R.check_o(got, ref[:, t][:, plain], mag[:, t][:, plain], slack[:, t], f"{name}: sequence {b} token {t}", p_step(case))
        if weights:
            R.check_w(cache.weight[b, :, :n], w, slack, f"{name}: weights of sequence {b}")


@pytest.mark.parametrize("name", CALLS)
def test_visible_values_near_the_largest(B, name):  # noqa: F811
    """V of up to 2^126 where a tile's logits lie above all earlier ones: no partial sum may leave fp32.  Per row at most
    four such values are visible, of one sign in a column, so that sum_j p_ij |v_j| < 2^128 for any p_ij <= 1."""
    case = CALLS[name]
    lens, P = case[5], case[9]
    cache, prefix, q = make(B, case, 70)
    q[:] = q[:, :1, :1]                                      # one direction for every row of a sequence ...
    if P:
        q[:] = q[:1]                                         # ... and for all that share the prefix
    scale = 1.0 / np.sqrt(128.0)

    def lift(k, n, qb):
        """Logits of 0, but in the last quarter of the slots 10 (base e), 14.4 in base 2."""
        if n < 4:
            return
        d = qb[0, 0].float()
        k[:, :n] = 0.1 * k[:, :n]
        k[:, n - n // 4:n] = (k[:, n - n // 4:n].float() + d * (10.0 / scale / float(d @ d))).to(torch.bfloat16)
    big = 2.0 ** 126
    for b, n in enumerate(lens):
        lift(cache.k[b], n, q[b])
        if n >= 4:
            cache.v[b, :, n - 1, 3] = big
            cache.v[b, :, n - n // 4, 4] = -big
            cache.v[b, :, 0, 5] = big
    if P:
        lift(prefix.k[0], P, q[0])
        prefix.v[0, :, P - 1, 3] = big
        prefix.v[0, :, P - P // 4 + 1, 4] = -big
        prefix.v[0, :, 0, 6] = big
    o = run(B, case, cache, prefix, q)
    for b, n, (ref, w, mag, slack) in wanted(case, cache, prefix, q):
        R.check_o(o[b], ref, mag, slack, f"{name}: sequence {b}", p_step(case))


@pytest.mark.parametrize("flip", [False, True], ids=["rising", "falling"])
def test_large_values_behind_a_prefix_whose_logits_outgrow_their_first_tile(B, flip):  # noqa: F811
    """160 rows: logits that rise by 60 (base 2) over the tiles that one workgroup takes, times V of 2^100."""
    P, batch = 20480, 20
    cache = cache_of(B, 80, batch, 8, 32, [1 + i for i in range(batch)], weight=False)
    q = queries(80, batch, 64, 1)
    q[:] = q[:1, :1]
    d = q[0, 0, 0].float()
    ramp = torch.arange(P, device="cuda") % 640 / 640.0 * 60.0 * float(np.log(2.0)) * float(np.sqrt(128.0)) / float(d @ d)
    if flip:
        ramp = ramp.flip(0)
    k = (ramp[:, None] * d[None]).to(torch.bfloat16).expand(1, 8, P, 128)
    g = torch.Generator("cuda").manual_seed(80)
    v = (torch.randn(1, 8, P, 128, generator=g, device="cuda") * 2.0 ** 100).to(torch.bfloat16)
    prefix = B.KVCache(k, v, torch.tensor([P], dtype=torch.int32, device="cuda"))
    o = torch.full_like(q, float("nan"))
    B.minf_prefix_attn(q, o, prefix, cache, workspace(B.minf_prefix_attn_workspace_bytes(q, prefix, cache)))
    torch.cuda.synchronize()
    pk, pv = R.f64(k)[0], R.f64(v)[0]
    qd, kd, vd = R.f64(q), R.f64(cache.k), R.f64(cache.v)
    for b in (0, 7, 19):
        heads = slice(0, 64, 8)                              # one query head of each group: all rows are alike
        ref, _, mag, slack = R.attention(qd[b][heads], kd[b], vd[b], 1 + b, 0, BIG, None, pk, pv)
        R.check_o(o[b][heads], ref, mag, slack, f"sequence {b}", R.P_BF16)


@pytest.mark.parametrize("batch", [2, 10, 25, 40], ids=lambda b: f"{4 * b}-rows")
def test_logits_of_minus_infinity_beside_very_low_ones(B, batch):  # noqa: F811
    """Keys whose logits are -inf have no weight, also where they fill whole tiles and parts and all other logits lie at
    -400 (base 2): the row is the softmax of those."""
    P, hkv = 9000, 8
    cache = cache_of(B, 90, batch, hkv, 32, [1 + i % 32 for i in range(batch)], weight=False)
    prefix = cache_of(B, 91, 1, hkv, P + 20, [P], weight=False)
    q = queries(90, batch, 4 * hkv, 1)
    q[:] = q[:1, :1]
    q[..., 0] = 1.0
    d = q[0, 0, 0].float()
    low = d * (-400.0 * float(np.log(2.0)) * float(np.sqrt(128.0)) / float(d @ d))
    prefix.k[:, :, :P] = (0.1 * prefix.k[:, :, :P].float() + low).to(torch.bfloat16)
    cache.k.copy_((0.1 * cache.k.float() + low).to(torch.bfloat16))
    prefix.k[:, :, 1000:4000, 0] = float("-inf")
    o = torch.full_like(q, float("nan"))
    B.minf_prefix_attn(q, o, prefix, cache, workspace(B.minf_prefix_attn_workspace_bytes(q, prefix, cache)))
    torch.cuda.synchronize()
    left = np.r_[0:1000, 4000:P]
    pk, pv = R.f64(prefix.k)[0][:, left], R.f64(prefix.v)[0][:, left]
    qd, kd, vd = R.f64(q), R.f64(cache.k), R.f64(cache.v)
    for b in (0, batch - 1):
        ref, _, mag, slack = R.attention(qd[b][::4], kd[b], vd[b], 1 + b % 32, 0, BIG, None, pk, pv)
        R.check_o(o[b][::4], ref, mag, slack, f"sequence {b}", R.P_BF16 if 4 * batch > 64 else R.P_TWO_BF16)
