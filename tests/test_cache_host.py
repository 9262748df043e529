"""The cache calls without a GPU: their refusals (nothing is enqueued then), the workspace sizes and how the
work is cut."""
import ctypes
import os
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2407_02490_amd", "libminf.so")
OK, NULL, SHAPE, BUDGET, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5
GB = 1 << 30


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(LIB):
        import __graft_entry__ as g
        g.build()
    from paper_2407_02490_amd import binding
    return binding.lib()


def cache(batch=2, heads=2, cap=1000, at=16 * GB, /, **kw):
    """Addresses are never dereferenced on the host."""
    from paper_2407_02490_amd.binding import _KVCache
    c = _KVCache()
    n = batch * heads * cap
    c.k, c.v, c.weight, c.lens = at, at + GB, at + 2 * GB, at + 3 * GB
    c.k_stride[:] = c.v_stride[:] = (heads * cap * 128, cap * 128, 128)
    c.weight_stride[:] = (heads * cap, cap)
    c.batch, c.n_kv_heads, c.capacity, c.head_dim = batch, heads, cap, 128
    assert n * 256 < GB
    for name, v in kw.items():
        if name.endswith("stride"):
            getattr(c, name)[:] = v
        else:
            setattr(c, name, v)
    return c


def queries(heads=4, n_new=1, /, **kw):
    from paper_2407_02490_amd.binding import _Queries
    x = _Queries()
    x.q, x.o = GB, 2 * GB
    x.q_stride[:] = x.o_stride[:] = (heads * n_new * 128, n_new * 128, 128)
    x.n_q_heads, x.n_new, x.softmax_scale = heads, n_new, 0.0
    for name, v in kw.items():
        if name.endswith("stride"):
            getattr(x, name)[:] = v
        else:
            setattr(x, name, v)
    return x


REF = ctypes.byref
WS = ctypes.c_void_p(8 * GB)


def attn(L, x, c, n_init=0, n_local=10, weights=0, ws=WS, nbytes=0):
    """Refused for what is wrong with the arguments, or, where nothing is, for the workspace (status 4)."""
    return L.minf_cache_attn(REF(x), REF(c), n_init, n_local, weights, ws, nbytes, None)


def test_cache_attn_refuses(L):
    x, c = queries(), cache()
    assert attn(L, x, c) == WORKSPACE                                   # all else is right
    assert attn(L, x, c, ws=None, nbytes=GB) == WORKSPACE
    assert attn(L, x, c, ws=ctypes.c_void_p(8 * GB + 128), nbytes=GB) == WORKSPACE
    assert L.minf_cache_attn(None, REF(c), 0, 1, 0, WS, GB, None) == NULL
    assert L.minf_cache_attn(REF(x), None, 0, 1, 0, WS, GB, None) == NULL
    for name in ("k", "v", "lens"):
        assert attn(L, x, cache(**{name: None})) == NULL
    assert attn(L, x, cache(weight=None)) == WORKSPACE                  # not asked for
    assert attn(L, x, cache(weight=None), weights=1) == NULL
    for name in ("q", "o"):
        assert attn(L, queries(**{name: None}), c) == NULL
    for kw in (dict(head_dim=64), dict(batch=0), dict(n_kv_heads=0), dict(capacity=0), dict(k=16 * GB + 8), dict(v=16 * GB + 2),
               dict(lens=16 * GB + 1), dict(k_stride=(1 << 20, 1 << 18, 64)), dict(v_stride=(1 << 20, 1 << 18, 132)),
               dict(k_stride=(1 << 20, 1 << 18, (1 << 24) + 8)), dict(k_stride=(-8, 1 << 18, 128)), dict(n_kv_heads=3),
               dict(capacity=(1 << 29) + 1)):
        assert attn(L, x, cache(**kw)) == SHAPE, kw
    for kw in (dict(n_q_heads=0), dict(n_q_heads=3), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
               dict(softmax_scale=float("inf")), dict(q=GB + 8), dict(o=2 * GB + 2), dict(q_stride=(512, 128, 4)),
               dict(o_stride=(512, 128, 100)), dict(o_stride=(0, 128, 128)), dict(o_stride=(256, 128, 128))):
        assert attn(L, queries(**kw), c) == SHAPE, kw
    for kw in (dict(n_new=0), dict(n_new=65)):
        assert attn(L, queries(**kw), c) == BUDGET, kw
    assert attn(L, x, c, n_init=-1) == BUDGET and attn(L, x, c, n_local=0) == BUDGET
    assert attn(L, x, c, weights=3) == UNSUPPORTED and attn(L, x, c, weights=-1) == UNSUPPORTED


def test_outputs_must_not_lie_over_inputs(L):
    x, c = queries(), cache()
    for where in (c.k, c.v, c.lens - 256, c.v + 999 * 256):
        assert attn(L, queries(o=where), c) == SHAPE
    assert attn(L, queries(o=x.q), c) == WORKSPACE                      # in the place of q
    assert attn(L, queries(o=x.q + 256), c) == SHAPE
    # a slice of the fused buffer that also holds K and V is apart from them
    fused = cache(k=16 * GB + 1024, v=16 * GB + 1536, k_stride=(1000 * 1024, 128, 1024), v_stride=(1000 * 1024, 128, 1024))
    assert attn(L, queries(q=16 * GB, o=16 * GB, q_stride=(1000 * 1024, 128, 1024), o_stride=(1000 * 1024, 128, 1024)), fused) == WORKSPACE
    assert attn(L, queries(o=c.weight), c) == WORKSPACE                 # not written, not read
    assert attn(L, queries(o=c.weight), c, weights=1) == SHAPE
    # weights of more than 16 rows per K/V head are computed from q when o is there already
    assert attn(L, queries(32, o=x.q), cache(), weights=1) == WORKSPACE
    assert attn(L, queries(34, o=x.q), cache(), weights=1) == SHAPE
    assert attn(L, queries(34, o=x.q), cache()) == WORKSPACE
    for where in (c.k, c.v + 256, x.q, c.lens):
        assert attn(L, x, cache(weight=where), weights=1) == SHAPE and attn(L, x, cache(weight=where)) == WORKSPACE
    for stride in ((0, 1000), (2000, 999), (1000, 1000), (2000, 0)):
        assert attn(L, x, cache(weight_stride=stride), weights=2) == SHAPE, stride
    assert attn(L, x, cache(weight_stride=(1000, 2000)), weights=2) == WORKSPACE


def test_prefix_attn_refuses(L):
    x, c = queries(), cache()

    def run(p, x=x, c=c):
        return L.minf_prefix_attn(REF(x), REF(p), REF(c), WS, 0, None)
    prefix = lambda **kw: cache(1, 2, 500, 32 * GB, **kw)
    assert run(prefix()) == WORKSPACE and run(prefix(weight=None)) == WORKSPACE
    assert L.minf_prefix_attn(REF(x), None, REF(c), WS, GB, None) == NULL
    assert L.minf_prefix_attn(REF(x), REF(prefix()), None, WS, GB, None) == NULL
    assert run(prefix(k=None)) == NULL and run(prefix(lens=None)) == NULL
    for kw in (dict(batch=2), dict(n_kv_heads=1), dict(head_dim=96), dict(capacity=0), dict(k_stride=(0, 1 << 16, 120))):
        assert run(prefix(**kw)) == SHAPE, kw
    assert run(prefix(), queries(o=32 * GB)) == SHAPE
    assert run(prefix(), queries(n_new=65)) == BUDGET


def test_cache_evict_refuses(L):
    c = cache()

    def run(c=c, to=None, keep=100, n_init=4, n_recent=8, kept=ctypes.c_void_p(4 * GB), nbytes=0):
        return L.minf_cache_evict(REF(c), n_init, n_recent, keep, REF(c if to is None else to), kept, WS, nbytes, None)
    other = lambda cap=200, **kw: cache(2, 2, cap, 32 * GB, **kw)
    assert run() == WORKSPACE and run(to=other()) == WORKSPACE and run(to=other(100)) == WORKSPACE
    assert run(to=other(lens=c.lens)) == WORKSPACE
    assert run(kept=None) == NULL and run(c=cache(weight=None)) == NULL and run(to=other(weight=None)) == NULL
    assert L.minf_cache_evict(None, 0, 0, 1, REF(c), ctypes.c_void_p(4 * GB), WS, GB, None) == NULL
    assert L.minf_cache_evict(REF(c), 0, 0, 1, None, ctypes.c_void_p(4 * GB), WS, GB, None) == NULL
    for kw in (dict(keep=0), dict(keep=11), dict(n_init=-1), dict(n_recent=-1), dict(n_init=2 ** 31 - 1), dict(keep=1001)):
        assert run(**kw) == BUDGET, kw
    assert run(to=other(99)) == BUDGET
    for to in (other(batch=1), other(n_kv_heads=1), other(k_stride=(0, 200 * 128, 128)), other(v_stride=(400 * 128, 128, 128)),
               other(weight_stride=(0, 200)), other(k=c.v), other(v=c.k + 256), other(weight=c.k), other(k=c.weight),
               cache(v=40 * GB), cache(weight=40 * GB), cache(capacity=999), cache(k_stride=(1 << 20, 1 << 18, 128)),
               other(lens=c.lens + 4), other(lens=c.k)):
        assert run(to=to) == SHAPE
    for kept in (c.k, c.weight, c.lens, c.v + 512, 4 * GB + 2):
        assert run(kept=ctypes.c_void_p(kept)) == SHAPE
    assert run(to=other(), kept=ctypes.c_void_p(32 * GB)) == SHAPE
    # K and V move at the same time
    both = cache(v=c.k)
    assert run(c=both) == SHAPE and run(c=both, to=other()) == WORKSPACE and run(to=other(v=32 * GB)) == SHAPE
    assert run(to=other(weight=32 * GB)) == SHAPE
    fused = cache(k=16 * GB, v=16 * GB + 512, k_stride=(1000 * 512, 128, 512), v_stride=(1000 * 512, 128, 512))
    assert run(c=fused) == WORKSPACE                                    # in place in a fused token-major buffer
    # broadcast caches can be read, not evicted in place
    flat = cache(k_stride=(0, 1000 * 128, 128))
    assert run(c=flat) == SHAPE and run(c=flat, to=other()) == WORKSPACE


def test_workspace_sizes(L):
    x, c = queries(), cache()
    plain = L.minf_cache_attn_workspace_bytes(REF(x), REF(c), 0, 1000, 0)
    weights = L.minf_cache_attn_workspace_bytes(REF(x), REF(c), 0, 1000, 1)
    assert plain > 0 and weights - plain >= 2 * 2 * 1000 * 2 * 4          # sequences, heads, keys, rows: the logits
    window = L.minf_cache_attn_workspace_bytes(REF(x), REF(c), 4, 60, 1)
    assert plain < window < weights
    assert L.minf_cache_attn_workspace_bytes(REF(x), REF(c), 0, 0, 0) == 0
    assert L.minf_cache_attn_workspace_bytes(REF(x), None, 0, 1, 0) == 0
    assert L.minf_cache_attn_workspace_bytes(None, REF(c), 0, 1, 0) == 0
    p = cache(1, 2, 500, 32 * GB)
    assert L.minf_prefix_attn_workspace_bytes(REF(x), REF(p), REF(c)) > 0
    assert L.minf_prefix_attn_workspace_bytes(REF(x), REF(cache(2, 2, 500)), REF(c)) == 0
    assert L.minf_cache_evict_workspace_bytes(REF(c), 10) > 0
    assert L.minf_cache_evict_workspace_bytes(REF(c), 0) == 0
    # the list of tiles is counted in 32 bits: a broadcast batch beyond that is refused
    huge = cache(2, 2, 1000, k_stride=(0, 0, 128), v_stride=(0, 0, 128), weight=None)
    huge.batch, huge.n_kv_heads, huge.capacity = 8191, 8, 1 << 26
    assert L.minf_cache_attn_workspace_bytes(REF(queries(8)), REF(huge), 0, 1 << 26, 0) == 0
    assert L.minf_cache_attn_workspace_bytes(REF(queries(8)), REF(huge), 0, 1 << 12, 0) > 0
    huge.batch = 8192
    assert L.minf_cache_attn_workspace_bytes(REF(queries(8)), REF(huge), 0, 1 << 12, 0) == 0


def test_a_call_that_needs_no_memory_names_a_workspace_all_the_same(L):
    """0 is the answer to invalid arguments, and a workspace without bytes has no address."""
    x, c = queries(8, 16, q_stride=(1 << 14, 2048, 128), o_stride=(1 << 14, 2048, 128)), cache(2, 2, 40)      # 64 rows, one tile
    n = L.minf_cache_attn_workspace_bytes(REF(x), REF(c), 0, 40, 0)
    assert n > 0
    assert attn(L, x, c, 0, 40, 0, None, n) == WORKSPACE and attn(L, x, c, 0, 40, 0, WS, n - 1) == WORKSPACE


def test_binding_checks_its_tensors():
    import torch
    from paper_2407_02490_amd import binding as B
    k = torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16)
    lens = torch.zeros(2, dtype=torch.int32)
    assert B.KVCache(k, k, lens, torch.zeros(2, 2, 64)).c_struct().capacity == 64
    for bad in ((k.float(), k, lens, None), (k, k[:, :, :32], lens, None), (k, k, lens.long(), None), (k, k, lens[:1], None),
                (k, k, lens, torch.zeros(2, 2, 63)), (k, k, lens, torch.zeros(2, 2, 64).double()),
                (k, k, lens, torch.zeros(2, 64, 2).transpose(1, 2)), (k.transpose(2, 3), k.transpose(2, 3), lens, None)):
        with pytest.raises(AssertionError):
            B.KVCache(*bad)
    c = B.KVCache(k, k, lens)
    q = torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16)
    assert B.minf_cache_attn_workspace_bytes(q, c) > 0
    for bad in (q.float(), q[:1], q[..., :64]):
        with pytest.raises(AssertionError):
            B.minf_cache_attn_workspace_bytes(bad, c)


def test_every_visible_slot_is_walked_once():
    with tempfile.TemporaryDirectory() as tmp:
        exe = os.path.join(tmp, "cache_walk_check")
        cmd = ["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2407_02490_amd", "csrc"),
               os.path.join(ROOT, "tests", "cache_walk_check.cpp"), "-o", exe]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        r = subprocess.run([exe], capture_output=True, text=True)
        assert r.returncode == 0 and r.stdout.startswith("ok walks"), r.stdout[-2000:] + r.stderr[-2000:]
