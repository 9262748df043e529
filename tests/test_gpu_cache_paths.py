"""The cache calls on lists and caches so long that a worker takes many tiles of several segments and a part of a prefix
holds many, on the placements and joins of large batches, against the definition in 64 bits.  What a case is for (tiles
per worker, tiles per part, which kernel) follows from its shapes: the tests without a GPU compute it and compare it with
the library's workspace size, so that a case that came to take another path fails there."""
import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests.test_gpu_cache import evict_and_check

BIG = 2 ** 31 - 1
WORKERS = 1024


@pytest.fixture(scope="module")
def B():
    from paper_2407_02490_amd import binding
    binding.lib()
    return binding


def lens_of(batch, cap):
    """Long sequences with empty and short ones between them."""
    pattern = [cap, 0, cap - 1, 1, 33, cap - 7, 64, cap // 2 + 5, 2, cap]
    return [pattern[i % 10] for i in range(batch)]


class Case:
    def __init__(self, batch, hq, hkv, T, cap, n_init=0, n_local=BIG, P=0, lens=None):
        self.batch, self.hq, self.hkv, self.T, self.cap, self.P = batch, hq, hkv, T, cap, P
        self.n_init, self.n_local = n_init, n_local
        self.lens = lens if lens is not None else lens_of(batch, cap)
        self.rows = hq // hkv * T
        self.p_rows = batch * self.rows if P else 0
        self.p_cap = P + 20 if P else 0

    # ---- what the call does with it
    def tiles(self, n, tile):
        """Of a sequence of n tokens: tiles of the slots that some row sees."""
        first = max(0, n - self.T - min(self.n_local, self.cap) + 1) // tile
        sink = -(-min(self.n_init, n) // tile)
        return -(-n // tile) if first <= sink else sink + -(-n // tile) - first

    def share(self, row_tiles, p_row_tiles=0, p_tiles=0):
        """Places of the list (tiles, and two per segment) that a worker takes."""
        own = sum(self.tiles(n, 32) + 2 for n in self.lens if n > 0)
        return -(-self.hkv * (row_tiles * own + p_row_tiles * (p_tiles + 2 if p_tiles else 0)) // WORKERS)

    def max_tiles(self):
        seen = min(min(self.n_init, self.cap) + min(self.n_local, self.cap) + self.T + 128, self.cap)
        return -(-seen // 32)

    def workspace(self, weights, block, row_tiles, p_row_tiles, slot_rows, shared):
        """Bytes: pieces of the workers (block: their rows), of shared parts (row tiles and parts, rows of a tile), weights."""
        up = lambda n: -(-n // 256) * 256
        segments = self.hkv * (self.batch * row_tiles + p_row_tiles)
        slots = (2 * WORKERS + segments) * slot_rows if segments else 0
        n = up(slots * 512) + up(slots * 8)
        for items, tile_rows in shared:
            n += up(items * tile_rows * 512) + up(items * tile_rows * 8)
        heads = self.batch * self.hkv
        if weights:
            n += up(heads * self.rows * 8)
            if self.rows <= 16:
                n += up(heads * self.max_tiles() * self.rows * 128)
        return max(n, 256)

    def tensors(self, device):
        """q, one K/V for all sequences (batch stride 0), the prefix."""
        kv = [torch.empty(1, self.hkv, self.cap, 128, dtype=torch.bfloat16, device=device) for _ in range(2)]
        pre = [torch.empty(1, self.p_cap, self.hkv, 128, dtype=torch.bfloat16, device=device).transpose(1, 2) for _ in range(2)] if self.P else None
        q = torch.empty(self.batch, self.hq, self.T, 128, dtype=torch.bfloat16, device=device)
        w = torch.empty(self.batch, self.hkv, self.cap, device=device)
        return q, kv, pre, w

    def caches(self, B, kv, pre, w, device):
        lens = torch.tensor(self.lens, dtype=torch.int32, device=device)
        cache = B.KVCache(*(t.expand(self.batch, -1, -1, -1) for t in kv), lens, w)
        prefix = B.KVCache(*pre, torch.tensor([self.P], dtype=torch.int32, device=device)) if self.P else None
        return cache, prefix

    def bytes(self, B, weights):
        q, kv, pre, w = self.tensors("cpu")
        cache, prefix = self.caches(B, kv, pre, w, "cpu")
        if self.P:
            return B.minf_prefix_attn_workspace_bytes(q, prefix, cache)
        return B.minf_cache_attn_workspace_bytes(q, cache, self.n_init, self.n_local, weights)


# workers (one wave each): 1 to 16 rows in one block, 17 to 32 of ragged batches and of prefixes in two
WORKER_CASES = {
    "1-row": Case(30, 8, 8, 1, 6000),
    "4-rows": Case(30, 32, 8, 1, 6000),
    "4-rows-window": Case(30, 32, 8, 1, 6000, 100, 2500),
    "4-rows-of-1280": Case(40, 32, 8, 1, 6000),             # more than 1024 rows in all: a wave each in the join
    "7-rows-of-2100": Case(75, 28, 4, 1, 4000),
    "16-rows": Case(30, 32, 8, 4, 6000),
    "16-rows-window": Case(30, 32, 8, 4, 6000, 33, 2500),
    "20-rows": Case(30, 32, 8, 5, 6000),
    "32-rows": Case(30, 32, 8, 8, 6000),
}
PREFIX_WORKER_CASES = {
    "8-rows": Case(2, 32, 8, 1, 700, P=45001, lens=[700, 333]),
    "16-rows": Case(4, 32, 8, 1, 700, P=45001, lens=[700, 1, 0, 333]),
    "32-rows": Case(4, 64, 8, 1, 700, P=45001, lens=[700, 1, 0, 333]),
    "24-rows": Case(3, 32, 8, 2, 3000, P=45001, lens=[3000, 1, 2999]),
}
# rows of a workgroup's tile, what it is for
SHARED_CASES = {
    "40-rows": (64, Case(16, 32, 4, 5, 6000)),
    "20-rows-window": (64, Case(12, 32, 8, 5, 6000, 100, 2500)),
    "64-rows-window": (64, Case(12, 32, 8, 16, 6000, 100, 2500)),
    "100-rows": (128, Case(8, 16, 4, 25, 6000)),
    "100-rows-window": (128, Case(16, 16, 4, 25, 6000, 100, 2500)),
    "200-rows": (128, Case(6, 32, 4, 25, 6000)),
    "100-rows-many": (128, Case(40, 32, 8, 25, 2000)),      # more workgroups than CUs
    "128-rows-many-window": (128, Case(40, 32, 8, 32, 4000, 40, 1500)),
}
SHARED_PREFIX_CASES = {
    "40-rows": (64, Case(10, 32, 8, 1, 300, P=70001)),
    "64-rows": (64, Case(16, 32, 8, 1, 300, P=69952)),
    "100-rows": (128, Case(25, 32, 8, 1, 300, P=70001)),
    "128-rows": (128, Case(4, 32, 8, 8, 300, P=70040)),
    "160-rows": (256, Case(40, 32, 8, 1, 300, P=21001)),
    "640-rows": (256, Case(40, 32, 8, 4, 300, P=83007)),
}
MODES = [None, "set", "add"]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("name", WORKER_CASES)
def test_worker_cases_take_many_tiles(B, name, mode):
    c = WORKER_CASES[name]
    block = 16 if c.rows <= 16 else 32
    assert c.share(1) >= 10
    assert c.bytes(B, mode) == c.workspace(mode, block, 1, 0, c.rows, [])


@pytest.mark.parametrize("name", PREFIX_WORKER_CASES)
def test_prefix_worker_cases_take_many_tiles(B, name):
    c = PREFIX_WORKER_CASES[name]
    block = 16 if c.p_rows <= 16 else 32
    assert c.share(1, 1, -(-c.P // 32)) >= 10
    assert c.bytes(B, None) == c.workspace(None, block, 1, 1, block, [])


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("name", SHARED_CASES)
def test_shared_cases_take_many_tiles(B, name, mode):
    tile_rows, c = SHARED_CASES[name]
    row_tiles = -(-c.rows // tile_rows)
    items = c.batch * c.hkv * row_tiles
    splits = [s for s in range(1, 65) if c.bytes(B, mode) == c.workspace(mode, 0, 0, 0, 0, [(items * s, tile_rows)] if s > 1 else [])]
    assert len(splits) == 1 and -(-c.tiles(c.cap, 64) // splits[0]) >= 9, splits
    assert ("many" in name) == (items * splits[0] > 256)


@pytest.mark.parametrize("name", SHARED_PREFIX_CASES)
def test_shared_prefix_cases_take_many_tiles(B, name):
    tile_rows, c = SHARED_PREFIX_CASES[name]
    row_tiles = -(-c.p_rows // tile_rows)
    block = 16
    p_rest = -(-c.p_rows // block) if tile_rows == 256 else 0
    splits = [s for s in range(1, 65)
              if c.bytes(B, None) == c.workspace(None, block, -(-c.rows // block), p_rest, block, [(c.hkv * row_tiles * s, tile_rows)])]
    if c.rows > 16:                                          # own rows: two blocks of them
        splits = [s for s in range(1, 65) if c.bytes(B, None) == c.workspace(None, 32, -(-c.rows // 32), p_rest, 32, [(c.hkv * row_tiles * s, tile_rows)])]
    assert len(splits) == 1 and c.P // 64 // splits[0] >= 9, splits


# ------------------------------------------------------------------ on the GPU
def fill(c, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    q, kv, pre, w = c.tensors("cuda")
    q.copy_(torch.randn(q.shape, generator=gen, device="cuda") * 1.5)
    longest = max(c.lens)
    for t in kv:
        t.normal_(generator=gen)
        t[:, :, longest:] = float("nan")
    for t in pre or []:
        t.normal_(generator=gen)
        t[:, :, c.P:] = float("nan")
    return q, kv, pre, w


def reference(c, q, kv, pre, b, h):
    """R.attention of the rows of one sequence and K/V head (its error terms are explained there), by torch in 64 bits."""
    n, group, scale = c.lens[b], c.hq // c.hkv, 1.0 / np.sqrt(128.0)
    qd = q[b, h * group:(h + 1) * group].double().reshape(-1, 128)
    k, v = kv[0][0, h, :n].double(), kv[1][0, h, :n].double()
    i = n - c.T + torch.arange(c.T, device="cuda")[:, None]
    j = torch.arange(n, device="cuda")[None]
    sees = (j <= i) & ((j < c.n_init) | (i - j < c.n_local))
    if pre is not None:
        k, v = torch.cat([pre[0][0, h, :c.P].double(), k]), torch.cat([pre[1][0, h, :c.P].double(), v])
        sees = torch.cat([(i >= 0).expand(-1, c.P), sees], 1)
    sees = sees.repeat(group, 1)
    s = (qd @ k.t()) * scale
    s = s.masked_fill(~sees, float("-inf"))
    top = s.amax(1, keepdim=True) if s.shape[1] else torch.zeros(len(qd), 1, dtype=torch.float64, device="cuda")
    p = torch.exp(s - torch.where(top.isinf(), 0.0, top))
    total = p.sum(1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    terms = (qd.abs() @ k.abs().t()).masked_fill(~sees, 0.0).amax(1) * scale if s.shape[1] else total[:, 0] * 0
    slack = 2 * (128 + 3) * 2.0 ** -24 * terms + (sees.sum(1) + 16) * 2.0 ** -23
    shape = lambda t: t.reshape(group, c.T, -1).cpu().numpy()
    return shape(p @ v), shape(p @ v.abs()), shape(slack[:, None])[..., 0], p[:, c.P:].sum(0).cpu().numpy()


def check(c, q, kv, pre, o, before=None, after=None, p_step=None):
    if p_step is None:
        p_step = R.P_BF16 if (c.p_rows or c.rows) > 64 else R.P_TWO_BF16
    group = c.hq // c.hkv
    for b, n in enumerate(c.lens):
        for h in range(c.hkv):
            want, mag, slack, w = reference(c, q, kv, pre, b, h)
            what = f"sequence {b} ({n} tokens) head {h}"
            R.check_o(o[b, h * group:(h + 1) * group], want, mag, slack, what, p_step)
            if before is None:
                continue
            got, old = after[b, h].double().cpu().numpy(), before[b, h].double().cpu().numpy()
            assert (got[n:] == old[n:]).all(), f"{what}: slots behind the sequence are left as they are"
            # the sums of p, in the order of the kernels: one rounding per row; adding rounds once more
            bound = w * (slack.max(initial=0.0) + (slack.size + 1) * 2.0 ** -24) + 2.0 ** -24 * np.abs(got[:n]) + 1e-30
            over = np.abs(got[:n] - old[:n] - w) / bound
            assert over.max(initial=0.0) <= 1.0, f"{what}: weights {over.max():.3g} times their bound"


def attend(B, c, q, kv, pre, w, mode):
    cache, prefix = c.caches(B, kv, pre, w, "cuda")
    o = torch.full_like(q, float("nan"))
    if prefix is not None:
        need = B.minf_prefix_attn_workspace_bytes(q, prefix, cache)
    else:
        need = B.minf_cache_attn_workspace_bytes(q, cache, c.n_init, c.n_local, mode)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    if prefix is not None:
        B.minf_prefix_attn(q, o, prefix, cache, ws)
    else:
        B.minf_cache_attn(q, o, cache, ws, n_init=c.n_init, n_local=c.n_local, weights=mode)
    torch.cuda.synchronize()
    return o


def run_own(B, c, mode, seed):
    q, kv, pre, w = fill(c, seed)
    w.uniform_(0.0, 2.0)
    before = w.clone()
    o = attend(B, c, q, kv, pre, w, mode)
    if mode is None:
        assert torch.equal(w, before)
    if mode == "set":                                        # what was there does not matter where a token is
        for b, n in enumerate(c.lens):
            before[b, :, :n] = 0.0
    check(c, q, kv, pre, o, before if mode else None, w)


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("name", WORKER_CASES)
def test_workers_of_many_tiles(B, name, mode):
    run_own(B, WORKER_CASES[name], mode, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("name", PREFIX_WORKER_CASES)
def test_workers_of_many_tiles_of_a_prefix(B, name):
    c = PREFIX_WORKER_CASES[name]
    q, kv, pre, w = fill(c, 2)
    check(c, q, kv, pre, attend(B, c, q, kv, pre, w, None))


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("name", SHARED_CASES)
def test_parts_of_many_tiles(B, name, mode):
    run_own(B, SHARED_CASES[name][1], mode, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("name", SHARED_PREFIX_CASES)
def test_parts_of_many_tiles_of_a_prefix(B, name):
    c = SHARED_PREFIX_CASES[name][1]
    q, kv, pre, w = fill(c, 4)
    check(c, q, kv, pre, attend(B, c, q, kv, pre, w, None))


@pytest.mark.gpu
@pytest.mark.parametrize("flip", [False, True], ids=["rising", "falling"])
@pytest.mark.parametrize("name", ["40-rows", "100-rows", "160-rows"])
def test_logits_that_rise_inside_a_part_of_a_prefix(B, name, flip):
    """By 200 (base 2) over every 320 slots, five tiles: references are taken anew in later tiles, and the loop of 256 rows,
    which takes one only once, from a part's first tile, 160 below the largest at times, sums beyond its limit of 2^100
    and redoes the part."""
    c = SHARED_PREFIX_CASES[name][1]
    q, kv, pre, w = fill(c, 5)
    q[:] = q[:1, :1, :1]
    d = q[0, 0, 0].float()
    ramp = torch.arange(c.P, device="cuda") % 320 / 320.0 * 200.0 * float(np.log(2.0)) * float(np.sqrt(128.0)) / float(d @ d)
    if flip:
        ramp = ramp.flip(0)
    pre[0][:, :, :c.P] = (0.05 * pre[0][:, :, :c.P].float() + ramp[:, None] * d[None]).to(torch.bfloat16)
    check(c, q, kv, pre, attend(B, c, q, kv, pre, w, None))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), -3.3895313892515355e38])
@pytest.mark.parametrize("name", ["4-rows-window", "20-rows-of-one-token", "80-rows-of-one-token", "one-workgroup"])
def test_slots_between_sink_and_window_do_not_matter_to_one_token(B, name, bad):
    c = {"4-rows-window": WORKER_CASES["4-rows-window"],
         "20-rows-of-one-token": Case(3, 20, 1, 1, 6000, 77, 1000),
         "80-rows-of-one-token": Case(3, 80, 1, 1, 6000, 77, 1000),
         "one-workgroup": Case(3, 8, 2, 1, 2000, 37, 90)}[name]
    q, kv, pre, w = fill(c, 6)
    n = 5000 if c.cap > 2000 else 1901
    c = Case(c.batch, c.hq, c.hkv, 1, c.cap, c.n_init, c.n_local, lens=[n] * c.batch)
    clean = [t.clone() for t in kv]
    for t in kv:
        t[:, :, c.n_init:n - c.n_local] = bad
        t[:, :, n:] = bad
    for mode in MODES:
        w.fill_(1.0)
        o = attend(B, c, q, kv, pre, w, mode)
        check(c, q, clean, pre, o)
        if mode:
            assert (w[:, :, c.n_init:n - c.n_local] == (mode == "add")).all() and (w[:, :, n:] == 1.0).all()


# ------------------------------------------------------------------ evictions of many long rows
# rows that are and are not multiples and divisors of the eight XCDs: batch, heads
ROWS = [(1, 8), (2, 8), (1, 3), (4, 3), (1, 5), (3, 8), (1, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False], ids=["in-place", "to-another"])
@pytest.mark.parametrize("shape", ROWS, ids=[f"{b}x{h}" for b, h in ROWS])
def test_evict_many_long_rows(B, shape, in_place):
    batch, heads, cap, keep = *shape, 40000, 3001
    gen = torch.Generator("cuda").manual_seed(7)
    lens = torch.tensor([[40000, 33333, 2999, 36001][i % 4] for i in range(batch)], dtype=torch.int32, device="cuda")
    k, v = (torch.empty(batch, heads, cap, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    w = torch.empty(batch, heads, cap, device="cuda").exponential_(generator=gen)
    w[torch.rand(w.shape, generator=gen, device="cuda") < 0.1] = 0.0
    cache = B.KVCache(k, v, lens, w)
    to = None
    if not in_place:
        to = B.alloc_kv_cache(batch, heads, keep + 5)
        to.k.zero_(), to.v.zero_()
    evict_and_check(B, cache, keep, 17, 300, to)


@pytest.mark.gpu
def test_captured_calls_of_many_rows_and_long_rows(B):
    """Attention of 100 rows with weights, a prefix of 160 rows and an eviction of long rows in one graph and one workspace,
    one call after the other; replayed with other queries, weights and lengths between eager calls."""
    own, pre = SHARED_CASES["100-rows"][1], SHARED_PREFIX_CASES["160-rows"][1]
    q, kv, _, w = fill(own, 8)
    pq, pkv, pp, pw = fill(pre, 9)
    gen = torch.Generator("cuda").manual_seed(10)
    cache, _ = own.caches(B, kv, None, w, "cuda")
    branch, prefix = pre.caches(B, pkv, pp, pw, "cuda")
    keep = 3001
    long = B.KVCache(*(torch.empty(1, 8, 40000, 128, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2)),
                     torch.tensor([40000], dtype=torch.int32, device="cuda"), torch.zeros(1, 8, 40000, device="cuda"))
    need = max(B.minf_cache_attn_workspace_bytes(q, cache, weights="set"), B.minf_prefix_attn_workspace_bytes(pq, prefix, branch),
               B.minf_cache_evict_workspace_bytes(long, keep))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    to = [B.alloc_kv_cache(1, 8, keep) for _ in range(2)]
    for t in to:
        t.k.zero_(), t.v.zero_()
    outs = [[torch.zeros_like(q), torch.zeros_like(pq), torch.zeros(1, 8, keep, dtype=torch.int32, device="cuda")] for _ in range(2)]

    def step(i):
        B.minf_cache_attn(q, outs[i][0], cache, ws, weights="set")
        B.minf_prefix_attn(pq, outs[i][1], prefix, branch, ws)
        B.minf_cache_evict(long, keep, ws, outs[i][2], to=to[i], n_init=5, n_recent=77)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(0)
    for turn in range(4):
        q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
        pq.copy_(torch.randn(pq.shape, generator=gen, device="cuda"))
        long.weight.exponential_(generator=gen)
        long.lens.fill_([40000, 2000, 39999, 3002][turn])
        cache.lens.copy_(cache.lens.roll(1))
        prefix.lens.fill_([21001, 64, 0, 20000][turn])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs[0] + [w, to[0].k, to[0].v, to[0].weight, to[0].lens]]
        w.zero_()
        step(1)
        torch.cuda.synchronize()
        for b, n in enumerate(cache.lens.tolist()):          # slots behind the sequences are left as they were
            got[3][b, :, n:] = 0.0
        for i, (a, e) in enumerate(zip(got, outs[1] + [w, to[1].k, to[1].v, to[1].weight, to[1].lens])):
            bits = {torch.bfloat16: torch.int16, torch.float32: torch.int32}.get(a.dtype, a.dtype)
            assert torch.equal(a.view(bits), e.view(bits)), f"replay {turn}, output {i}"
