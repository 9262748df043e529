"""The Python calls of the cache without a GPU: integers beyond the library's 32 bits, which the binding must not cut."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2407_02490_amd import binding
    binding.lib()
    return binding


@pytest.fixture()
def cache(B):
    k = torch.zeros(2, 2, 1000, 128, dtype=torch.bfloat16)
    return B.KVCache(k, k.clone(), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 1000))


def test_windows_beyond_32_bits_are_the_whole_cache(B, cache):
    q = torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16)
    size = lambda n_init, n_local: B.minf_cache_attn_workspace_bytes(q, cache, n_init, n_local, "set")
    whole = size(0, None)
    assert size(0, 5) < whole
    for far in (1000, 2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 40, 10 ** 20):
        assert size(0, far) == whole and size(far, 5) == size(1000, 5)
    for n in (-1, -2 ** 31, -2 ** 32 + 5, -10 ** 20):
        assert size(n, 5) == 0 and size(0, n) == 0           # refused
    assert size(0, 0) == 0


def test_counts_beyond_32_bits_are_refused(B, cache, monkeypatch):
    seen = []
    monkeypatch.setattr(B, "_cache_call", lambda fn, c, ws, stream, *args: seen.append(args))
    kept = torch.zeros(2, 2, 100, dtype=torch.int32)
    B.minf_cache_evict(cache, 100, None, kept, n_init=2 ** 32 + 5, n_recent=-2 ** 32 + 7)
    B.minf_cache_attn(torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 1, 128, dtype=torch.bfloat16), cache, None,
                      n_init=2 ** 32 + 5, n_local=-2 ** 32 + 7)
    assert seen[0][1:4] == (2 ** 31 - 1, -1, 100) and seen[1][2:4] == (1000, -1)
    assert B.minf_cache_evict_workspace_bytes(cache, 100) > 0 and B.minf_cache_evict_workspace_bytes(cache, -2 ** 32 + 100) == 0
