"""The references of the cache's GPU tests against each other (CPU only)."""
import pytest
import torch

import test_gpu_cache as slow
import test_gpu_cache_wide as fast


@pytest.mark.parametrize("lens,keep,sink,recent,Hkv,page,dtype,kind", slow.EVICT[:8] + [
    ([900, 3], 400, 7, 50, 2, 16, slow.BF, "odd"), ([900, 3], 400, 500, 50, 2, 16, slow.BF, "odd")])
def test_eviction(lens, keep, sink, recent, Hkv, page, dtype, kind):
    """Whole arrays at a time as slot by slot."""
    pool, seen = fast.long_pool(None, lens, Hkv, page, dtype, kind, sink), [n + n // 2 for n in lens]
    K, V, W, S = (x.clone() for x in (pool.K, pool.V, pool.W, pool.S))
    left = slow.evict64(pool, K, V, W, S, seen, keep, sink, recent)
    k, v, w, s, n = fast.evict64(pool, seen, keep, sink, recent)
    assert n == left and torch.equal(K, k) and torch.equal(V, v) and torch.equal(S, s)
    assert torch.equal(W.view(torch.int32), w.view(torch.int32))


@pytest.mark.parametrize("causal", [False, True])
def test_attention(causal):
    """All rows under a mask as row by row, also with values, keys and logits that are not finite."""
    import numpy as np
    q, k, v = (slow.normal(i, (n, 64), slow.F32) for i, n in ((1, 50), (2, 90), (3, 90)))
    v[60, 5], v[70, 6], k[80, 0], k[85, 1], k[10, 2] = float("nan"), float("inf"), float("nan"), float("inf"), float("-inf")
    vis = 90 - 50 + np.arange(50) + 1 if causal else np.full(50, 90)
    sees = torch.arange(90) < torch.from_numpy(vis)[:, None]
    for keys in (k, torch.where(torch.isfinite(k), k, 0.0)):
        want = slow.attend64(q, keys, v, vis)
        got = fast.whole64(q, keys, v, sees, 0.125)
        for i, (x, y) in enumerate(zip(want[:3], got[:3])):
            x = torch.from_numpy(x)
            assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(torch.isinf(x), torch.isinf(y)), i
            fin = torch.isfinite(x)
            assert torch.allclose(x[fin], y[fin], rtol=1e-12, atol=1e-14), i
