"""More of the paged key-value cache on the GPU against the 64-bit computations of test_gpu_cache.py, with
its tolerances: u = 2^-24, a row's E, one bf16 rounding up to 2^-8 of a value."""
import pytest
import torch

from test_gpu_cache import BF, F32, Pool, _gpu, cache, check_attend, gen, log, normal  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,causal", [
    ([200], [1], 2, 2, 16, BF, True), ([9000, 40], [1, 1], 4, 1, 64, BF, True), ([9000, 40], [1, 1], 4, 1, 64, F32, True),
    ([700], [40], 2, 1, 32, F32, True), ([700], [130], 2, 2, 32, BF, True), ([2000, 300], [150, 90], 2, 2, 16, F32, True),
    ([40000], [1], 1, 1, 256, BF, True), ([1374, 1374], [1374, 1374], 8, 8, 64, BF, False)])
def test_attend_values_near_the_largest(cache, lens, qs, Hq, Hkv, page, dtype, causal):  # noqa: F811
    """Values of 1e38 to 3e38 under flat logits: sums of them pass fp32's range, their means do not."""
    log("attend large values %s %s %s" % (lens, qs, dtype))
    pool = Pool(cache, lens, Hkv, page, dtype, seed=820 + sum(lens))
    for b, n in enumerate(lens):
        v = (1e38 + 2e38 * torch.rand(n, Hkv, 64, generator=gen(b))) * torch.tensor([1.0, -1.0]).repeat(32)
        v[:, :, :4] = normal(821 + b, (n, Hkv, 4), F32).clamp(-3, 3) * 1e38     # of either sign in the first features
        pool.put(b, pool.k[b], v.to(dtype))
    check_attend(cache, pool, normal(822, (sum(qs), Hq, 64), dtype), qs, causal)
