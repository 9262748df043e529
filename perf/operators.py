"""The calls by which the cache operators are judged: what a serving program does
with the keys and values that a long prefill leaves behind.

  window   one decode step of A-shape heads: sink + sliding window over a cache
  weights  one decode step that also gives every cached key the attention weight
           it received (the input of an eviction)
  prefix   one decode step of a batch whose sequences share a long prefix
  evict    a cache reduced to the keys of largest weight

`own` chooses between the plain form (elementary torch operations in 32 bits)
and the calls of this library.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128

# Shape of one call; listed() and draw() override what differs.  `lens` says how the sequence
# lengths of a batch are spread: "full" (the capacity), "near" (its last tenth), "ragged" (one token up
# to the capacity, evenly in the logarithm).
_BASE = dict(kind="window", B=1, hq=32, kv=8, T=1, cap=8192, lens="near", layout="head",
             n_init=1024, n_local=4096, P=0, keep=0, n_recent=0)


def _case(**kw):
    c = dict(_BASE)
    c.update(kw)
    return c


def listed():
    return [
        # one sequence, one token, the default sink + window: the smallest call, where latency counts
        _case(name="window-one"),
        # a serving batch of unequal lengths, from one token on
        _case(name="window-ragged", B=32, cap=32768, lens="ragged"),
        # five drafted tokens at a time, one K/V head for eight query heads, token-major cache, odd window
        _case(name="window-draft", B=6, hq=8, kv=1, T=5, cap=16451, lens="ragged", layout="token",
              n_init=100, n_local=1000),
        # short chats: two sequences of up to 2K tokens, weights of every key
        _case(name="weights-short", kind="weights", B=2, cap=2048),
        # two prompts of 128K tokens, the default layer
        _case(name="weights-128k", kind="weights", B=2, cap=131072),
        # one prompt of a million tokens: the largest cache
        _case(name="weights-1m", kind="weights", cap=1048576, lens="full"),
        # the last 64 rows of a prompt weigh its keys before the first eviction
        _case(name="weights-observe", kind="weights", hq=16, kv=4, T=64, cap=40256, lens="full"),
        # four answers to one short prompt
        _case(name="prefix-few", kind="prefix", B=4, P=4096, cap=512, lens="ragged"),
        # a batch of questions on one document of 128K tokens
        _case(name="prefix-128k", kind="prefix", B=32, P=131072, cap=2048, lens="ragged"),
        # many samples of one prompt of an odd length: the prefix is matrix work here
        _case(name="prefix-many", kind="prefix", B=160, P=20031, cap=1024, lens="ragged"),
        # four prompts of ragged lengths down to 4K keys each
        _case(name="evict-40k", kind="evict", B=4, kv=4, cap=40256, keep=4096, n_init=16, n_recent=256),
        # a million tokens down to 16K, token-major cache
        _case(name="evict-1m", kind="evict", cap=1048576, lens="full", layout="token", keep=16384,
              n_init=64, n_recent=1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window", "window", "weights", "weights", "prefix", "prefix", "evict"])
    kv = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 4, 7, 8])
    c = _case(kind=kind, kv=kv, hq=kv * group, lens=rng.choice(["full", "near", "ragged", "ragged"]),
              layout=rng.choice(["head", "head", "token"]))
    # as many sequences as keep the caches within 2M tokens of one K/V head ...
    c["cap"] = _log(rng, 64, 524288 if kind != "prefix" else 8192)
    c["B"] = _log(rng, 1, max(1, min(128, (1 << 21) // (c["cap"] * kv))))
    # ... one token in two of three calls, drafted tokens or a piece of a prompt otherwise
    c["T"] = rng.choice([1, 1, 1, 1, rng.randint(2, 16), rng.randint(17, 64)])
    if kind == "window":
        c["n_init"], c["n_local"] = rng.choice([(1024, 4096), (128, 1024), (100, 1000), (4, 2044), (0, 512), (0, 1)])
    if kind == "prefix":
        c["P"] = _log(rng, 64, 262144)
        c["T"] = min(c["T"], 8)
        while c["B"] * c["T"] * c["hq"] * c["P"] > 1 << 27:
            c["B"], c["P"] = max(1, c["B"] // 2), max(64, c["P"] // 2)
    # ... and no more matrix work than the largest listed call
    while c["B"] * c["T"] * c["hq"] * c["cap"] > 1 << 27:
        c["T"], c["B"] = (c["T"] // 2, c["B"]) if c["T"] > 1 else (1, c["B"] // 2)
    if kind == "evict":
        c["T"] = 1
        c["keep"] = _log(rng, 16, c["cap"])
        c["n_recent"] = rng.randint(0, c["keep"] // 2)
        c["n_init"] = rng.randint(0, min(64, c["keep"] // 2))
    return c


def _lens(case):
    """Sequence lengths: part of the case, not of the seed."""
    B, cap = case["B"], case["cap"]
    rng = random.Random(f"{B} {cap} {case['kv']} {case['kind']}")
    if case["lens"] == "full":
        return [cap] * B
    if case["lens"] == "near":
        return [rng.randint(max(1, cap - cap // 10), cap) for _ in range(B)]
    return [min(cap, _log(rng, 1, cap)) for _ in range(B)]


def _visible(case, n):
    """Keys of a sequence of n tokens that some row of a window call sees."""
    if case["kind"] != "window":
        return n
    first = max(0, n - case["T"] + 1 - case["n_local"])
    return min(n, case["n_init"]) + n - max(first, min(n, case["n_init"]))


def work(case):
    B, hq, kv, T = case["B"], case["hq"], case["kv"], case["T"]
    lens = _lens(case)
    if case["kind"] == "evict":
        kept = sum(min(n, case["keep"]) for n in lens)
        return {"bytes": kv * (4 * sum(lens) + kept * (2 * (4 * D + 4) + 4)), "flops": 0}
    keys = sum(_visible(case, n) for n in lens)
    nbytes = kv * 4 * D * (keys + case["P"]) + B * T * hq * D * 4
    if case["kind"] == "weights":
        nbytes += 4 * kv * sum(lens)
    return {"bytes": nbytes, "flops": 4 * D * T * hq * (keys + B * case["P"])}


# ------------------------------------------------------------------ inputs
def _cache_tensor(case, lead, n, gen):
    """[*lead, heads, n, 128] standard normal bf16, head-major or a view of token-major storage."""
    kv = case["kv"]
    if case["layout"] == "token":
        t = torch.empty(*lead, n, kv, D, dtype=torch.bfloat16, device="cuda")
        t.normal_(generator=gen)
        return t.transpose(-3, -2)
    t = torch.empty(*lead, kv, n, D, dtype=torch.bfloat16, device="cuda")
    return t.normal_(generator=gen)


def _plant(k, q, n, gen, count):
    """Adds 2 * the group's mean query direction to `count` of n keys: what attention sinks and the
    few heavy keys of trained models do to the logits.  k [kv, n, 128], q [hq, T, 128]."""
    kv, group = k.shape[0], q.shape[0] // k.shape[0]
    at = torch.randint(0, n, (count,), generator=gen, device="cuda")
    at[0] = 0
    mean = q.float().view(kv, group, -1, D).mean(dim=(1, 2))
    k[:, at] = (k[:, at].float() + 2.0 * mean[:, None]).to(torch.bfloat16)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed % (1 << 62))
    B, hq, kv, T, cap = case["B"], case["hq"], case["kv"], case["T"], case["cap"]
    lens = _lens(case)
    st = {"case": case, "k": _cache_tensor(case, (B,), cap, gen), "v": _cache_tensor(case, (B,), cap, gen),
          "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "host_lens": lens}
    if case["kind"] == "evict":
        # accumulated weights: a few heavy keys, a long tail, some keys that nothing looked at (ties)
        w = torch.empty(B, kv, cap, device="cuda").exponential_(generator=gen).pow_(4.0)
        w *= torch.rand(B, kv, cap, generator=gen, device="cuda") > 0.05
        st["weight"] = w
        room = case["keep"] + 64
        st["to_k"] = torch.zeros(B, kv, room, D, dtype=torch.bfloat16, device="cuda")
        st["to_v"] = torch.zeros_like(st["to_k"])
        st["to_weight"] = torch.zeros(B, kv, room, device="cuda")
        st["to_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        st["kept"] = torch.full((B, kv, case["keep"]), -1, dtype=torch.int32, device="cuda")
    else:
        st["q"] = torch.randn(B, hq, T, D, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)
        for b in range(B):
            _plant(st["k"][b], st["q"][b], lens[b], gen, 1 + lens[b] // 512)
        if case["kind"] == "weights":
            st["weight"] = torch.zeros(B, kv, cap, device="cuda")
        if case["kind"] == "prefix":
            st["pk"], st["pv"] = (_cache_tensor(case, (), case["P"], gen) for _ in range(2))
            _plant(st["pk"], st["q"].transpose(0, 1).reshape(hq, B * T, D), case["P"], gen, 1 + case["P"] // 512)
            st["plens"] = torch.tensor([case["P"]], dtype=torch.int32, device="cuda")
    if own:
        _handles(st)
    return st


def _handles(st):
    """The library's views of these tensors and the workspace, as a serving program keeps them."""
    from paper_2407_02490_amd import binding as lib
    case = st["case"]
    st["lib"] = lib
    st["cache"] = lib.KVCache(st["k"], st["v"], st["lens"], st.get("weight"))
    if case["kind"] == "evict":
        st["to"] = lib.KVCache(st["to_k"], st["to_v"], st["to_lens"], st["to_weight"])
        need = lib.minf_cache_evict_workspace_bytes(st["cache"], case["keep"])
    else:
        st["o"] = torch.empty_like(st["q"])
        if case["kind"] == "prefix":
            st["prefix"] = lib.KVCache(st["pk"][None], st["pv"][None], st["plens"])
            need = lib.minf_prefix_attn_workspace_bytes(st["q"], st["prefix"], st["cache"])
        elif case["kind"] == "window":
            need = lib.minf_cache_attn_workspace_bytes(st["q"], st["cache"], n_init=case["n_init"],
                                                       n_local=case["n_local"])
        else:
            need = lib.minf_cache_attn_workspace_bytes(st["q"], st["cache"], weights="set")
    st["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ one pass
def _run_own(st):
    case, lib = st["case"], st["lib"]
    if case["kind"] == "window":
        lib.minf_cache_attn(st["q"], st["o"], st["cache"], st["ws"], n_init=case["n_init"], n_local=case["n_local"])
        return {"o": st["o"]}
    if case["kind"] == "weights":
        lib.minf_cache_attn(st["q"], st["o"], st["cache"], st["ws"], weights="set")
        return {"o": st["o"], "weight": st["weight"]}
    if case["kind"] == "prefix":
        lib.minf_prefix_attn(st["q"], st["o"], st["prefix"], st["cache"], st["ws"])
        return {"o": st["o"]}
    lib.minf_cache_evict(st["cache"], case["keep"], st["ws"], to=st["to"], kept=st["kept"],
                         n_init=case["n_init"], n_recent=case["n_recent"])
    return {"k": st["to_k"], "v": st["to_v"], "weight": st["to_weight"], "lens": st["to_lens"], "kept": st["kept"]}


def _plain_rows(case, q, k, v, n, pk=None, pv=None):
    """Attention of one sequence: q [hq, T, 128], k/v [kv, cap, 128], n tokens.  Returns o and, per
    K/V head, the weights of the n keys."""
    hq, T, kv = q.shape[0], q.shape[1], k.shape[0]
    group = hq // kv
    i0 = n - T
    lo = max(0, i0 + 1 - case["n_local"]) if case["kind"] == "window" else 0
    sink = min(case["n_init"], lo) if case["kind"] == "window" else 0
    key = torch.cat([torch.arange(0, sink, device=q.device), torch.arange(lo, n, device=q.device)])
    kf = torch.cat([k[:, :sink], k[:, lo:n]], dim=1).float()
    vf = torch.cat([v[:, :sink], v[:, lo:n]], dim=1).float()
    row = i0 + torch.arange(T, device=q.device)
    seen = key[None, :] <= row[:, None]
    if case["kind"] == "window":
        seen &= (key[None, :] < case["n_init"]) | (row[:, None] - key[None, :] < case["n_local"])
    qf = q.float().reshape(kv, group * T, D)
    s = torch.matmul(qf, kf.transpose(1, 2)) * (1.0 / math.sqrt(D))
    s = s.masked_fill(~seen.repeat(group, 1)[None], float("-inf"))
    if pk is not None:
        s = torch.cat([torch.matmul(qf, pk.transpose(1, 2)) * (1.0 / math.sqrt(D)), s], dim=2)
        vf = torch.cat([pv, vf], dim=1)
    m = s.amax(dim=2, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), torch.zeros_like(m), m))
    total = p.sum(dim=2, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = torch.matmul(p, vf).reshape(hq, T, D)
    o = torch.where((row >= 0)[None, :, None], o, torch.zeros_like(o))
    return o.to(torch.bfloat16), p.sum(dim=1)


def _run_plain(st):
    case, lens = st["case"], st["host_lens"]
    if case["kind"] == "evict":
        return _evict_plain(st)
    o = torch.empty_like(st["q"])
    pk, pv = (st["pk"].float(), st["pv"].float()) if case["kind"] == "prefix" else (None, None)
    weight = torch.zeros_like(st["weight"]) if case["kind"] == "weights" else None
    for b, n in enumerate(lens):
        o[b], w = _plain_rows(case, st["q"][b], st["k"][b], st["v"][b], n, pk, pv)
        if weight is not None:
            weight[b, :, :n] = w
    return {"o": o} if weight is None else {"o": o, "weight": weight}


def _evict_plain(st):
    case = st["case"]
    keep, out = case["keep"], {}
    out["k"], out["v"] = torch.zeros_like(st["to_k"]), torch.zeros_like(st["to_v"])
    out["weight"], out["lens"] = torch.zeros_like(st["to_weight"]), torch.empty_like(st["to_lens"])
    out["kept"] = torch.full_like(st["kept"], -1)
    for b, n in enumerate(st["host_lens"]):
        w = st["weight"][b, :, :n]
        take = min(n, keep)
        if n > keep:
            score = w.clone()
            score[:, :case["n_init"]] = float("inf")
            score[:, n - case["n_recent"]:] = float("inf")
            at = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :keep]
            at = torch.sort(at, dim=1).values
        else:
            at = torch.arange(n, device="cuda").expand(w.shape[0], n)
        rows = at[:, :, None].expand(-1, -1, D)
        out["k"][b, :, :take] = st["k"][b].gather(1, rows)
        out["v"][b, :, :take] = st["v"][b].gather(1, rows)
        out["weight"][b, :, :take] = w.gather(1, at)
        out["lens"][b] = take
        out["kept"][b, :, :take] = at.to(torch.int32)
    return out


def run(st):
    return _run_own(st) if own else _run_plain(st)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_attention(st):
    case = st["case"]
    B, hq, kv, T = case["B"], case["hq"], case["kv"], case["T"]
    group = hq // kv
    o = torch.zeros(B, hq, T, D, dtype=torch.float64, device="cuda")
    weight = torch.zeros(B, kv, case["cap"], dtype=torch.float64, device="cuda")
    for h in range(kv):
        pk = st["pk"][h].double() if case["kind"] == "prefix" else None
        pv = st["pv"][h].double() if case["kind"] == "prefix" else None
        for b, n in enumerate(st["host_lens"]):
            kd, vd = st["k"][b, h, :n].double(), st["v"][b, h, :n].double()
            for t0 in range(0, T, 4):
                ts = [t for t in range(t0, min(T, t0 + 4)) if n - T + t >= 0]
                if not ts:
                    continue
                qd = st["q"][b, h * group:(h + 1) * group, ts].double()
                j = torch.arange(n, device="cuda")
                i = torch.tensor([n - T + t for t in ts], device="cuda")
                dist = i[:, None] - j[None, :]
                hidden = dist < 0
                if case["kind"] == "window":
                    hidden |= (dist >= case["n_local"]) & (j >= case["n_init"])[None, :]
                logit = (qd.reshape(-1, D) @ kd.T).view(group, len(ts), n) / math.sqrt(D)
                logit = logit.masked_fill(hidden, -math.inf)
                if pk is not None:
                    logit = torch.cat(((qd.reshape(-1, D) @ pk.T).view(group, len(ts), -1) / math.sqrt(D), logit), 2)
                logit -= torch.logsumexp(logit, dim=2, keepdim=True)
                p = torch.exp(logit)
                rows = p.reshape(group * len(ts), -1)
                if pk is None:
                    res = rows @ vd
                else:
                    res = rows[:, :pk.shape[0]] @ pv + rows[:, pk.shape[0]:] @ vd
                o[b, h * group:(h + 1) * group, ts] = res.view(group, len(ts), D)
                weight[b, h, :n] += rows[:, -n:].sum(dim=0)
    return {"o": o, "weight": weight} if case["kind"] == "weights" else {"o": o}


def _exact_evict(st):
    case = st["case"]
    out = {"k": torch.zeros(st["to_k"].shape, dtype=torch.float64),
           "v": torch.zeros(st["to_v"].shape, dtype=torch.float64),
           "weight": torch.zeros(st["to_weight"].shape, dtype=torch.float64),
           "lens": torch.zeros(st["to_lens"].shape, dtype=torch.int32),
           "kept": torch.full(st["kept"].shape, -1, dtype=torch.int32)}
    out = {name: t.cuda() for name, t in out.items()}
    for b, n in enumerate(st["host_lens"]):
        for h in range(case["kv"]):
            weight = st["weight"][b, h, :n].double().cpu().numpy()
            chosen = np.arange(n)
            if n > case["keep"]:
                first, last = case["n_init"], n - case["n_recent"]
                middle = np.arange(first, last)
                best = middle[np.lexsort((middle, -weight[first:last]))][:case["keep"] - first - case["n_recent"]]
                chosen = np.sort(np.concatenate([chosen[:first], best, chosen[last:]]))
            take = len(chosen)
            at = torch.from_numpy(chosen).cuda()
            out["kept"][b, h, :take] = at.to(torch.int32)
            out["weight"][b, h, :take] = torch.from_numpy(weight[chosen]).cuda()
            out["k"][b, h, :take] = st["k"][b, h].index_select(0, at).double()
            out["v"][b, h, :take] = st["v"][b, h].index_select(0, at).double()
        out["lens"][b] = min(n, case["keep"])
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_evict(st) if case["kind"] == "evict" else _exact_attention(st)
