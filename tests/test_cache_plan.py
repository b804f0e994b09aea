"""How the paged cache's attention divides a call, on the host: the plan's numbers agree with each other and with
the workspace, and the rules of its comment hold (CPU only: no call here launches a kernel)."""
import ctypes

import pytest

from paper_2609_23733_amd import vp
from test_cache_abi import R, batch, cache
from test_gpu_cache_wide import BF, WIDE


@pytest.fixture(scope="module")
def lib():
    return vp.load_library()


def plan(lib, Hq, c, b):
    p = vp.vp_cache_plan()
    code = lib.vp_cache_attend_plan(R(c), R(b), Hq, R(p))
    return code, p


def bounds(lens, qs, page, Hkv, dtype, **kw):
    n = max(lens)
    return (cache(Hkv=Hkv, page=page, dtype=vp.VP_BF16 if dtype else vp.VP_F32, npages=1 << 20, **kw),
            batch(B=len(lens), T=sum(qs), max_q=max(qs), max_len=n, max_pages=max(1, -(-n // page))))


@pytest.mark.parametrize("bf", [True, False])
def test_plan_adds_up(lib, bf):
    for B in (1, 3, 40):
        for q in (0, 1, 7, 64, 65, 300, 1374):
            for n in (0, 1, 63, 700, 5000, 44000):
                for Hq, Hkv in ((16, 16), (16, 4), (6, 2), (5, 1)):
                    c, b = bounds([n] * B, [q] * B, 64, Hkv, bf)
                    code, p = plan(lib, Hq, c, b)
                    assert code == 0
                    G, e = Hq // Hkv, p.range_slots
                    assert p.rows == (32 if not p.shared else 256 if bf else 128)
                    assert p.row_tiles == max(1, -(-q * G // p.rows))
                    assert e % 64 == 0 and e >= 64 and p.ranges >= 1 and p.ranges * e >= n > (p.ranges - 1) * e - 1
                    assert p.ranges <= 256 and (p.shared or not q * G > 64 or bf)
                    assert not (p.shared and q * G <= 64)
                    if p.logits_kept:
                        assert not p.shared and q * G <= (32 if bf else 64)
                    rows = b.T * Hq
                    parts = rows * p.ranges * 66 * 4 if p.ranges > 1 else 0
                    kept = rows * -(-n // 64) * 64 * 4 if p.logits_kept else rows * 4
                    size = lib.vp_cache_attend_workspace_bytes(R(c), R(b), Hq)
                    assert parts + kept <= size <= parts + kept + 4 * 256


@pytest.mark.parametrize("lens,qs,Hq,Hkv,page,dtype,causal", WIDE)
def test_plan_of_the_wide_cases(lib, lens, qs, Hq, Hkv, page, dtype, causal):
    code, p = plan(lib, Hq, *bounds(lens, qs, page, Hkv, dtype == BF))
    assert code == 0 and p.shared == 1


def test_plan_refusals(lib):
    p = vp.vp_cache_plan()
    assert lib.vp_cache_attend_plan(None, R(batch()), 8, R(p)) == 1
    assert lib.vp_cache_attend_plan(R(cache()), None, 8, R(p)) == 1
    assert lib.vp_cache_attend_plan(R(cache()), R(batch()), 8, None) == 1
    assert lib.vp_cache_attend_plan(R(cache()), R(batch()), 6, R(p)) == 1
    assert lib.vp_cache_attend_plan(R(cache(page=48)), R(batch()), 8, R(p)) == 2
    assert lib.vp_cache_attend_plan(R(cache()), R(batch(max_len=641)), 8, ctypes.byref(p)) == 1


def test_weights_need_the_queries_kept(lib):
    """The weights' kernel reads Q after O is written: the same tensor for both is refused with them."""
    from test_cache_abi import FAKE, attend
    assert attend(lib, cache(), batch(), Q=FAKE, O=FAKE, wo=FAKE) == 1
