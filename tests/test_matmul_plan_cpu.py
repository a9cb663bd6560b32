"""Which shape of workgroups a product takes, as the library states it, and that the products of the GPU tests meet every one."""
import numpy as np
import pytest

import paper_2510_08525_amd as rl
from matmul_shapes import SHAPES, lists


@pytest.mark.parametrize("dtype", [rl.RLKV_F32, rl.RLKV_BF16])
def test_every_shape_of_every_list_is_met(dtype):
    taken, lengths = lists(dtype)
    assert set(lengths) == {"sixteen", "sixty-four", "many"}
    for kind, length in lengths.items():
        assert sorted(taken[kind]) == list(range(length)), (kind, {at: len(s) for at, s in taken[kind].items()})


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [rl.RLKV_F32, rl.RLKV_BF16])
def test_they_are_ragged(m, n, k, dtype):
    bm, bn, parts, _, _ = rl.rlkv_plan_matmul(m, n, k, dtype)
    assert n % bn != 0 and (m % bm != 0 or m == 16 or m == 64) and k % 128 != 0 and k > 5 * 128
    assert bm in (16, 32, 64, 128, 192, 256) and bn in (16, 64, 128, 256) and parts in (1, 2, 4, 8)


@pytest.mark.parametrize("bad", [dict(m=0), dict(m=-1), dict(n=0), dict(k=0), dict(k=120), dict(dtype=2), dict(dtype=-1), dict(m=(1 << 24) + 1),
                                 dict(m=1 << 18, n=1 << 18), dict(plan=None)])
def test_refusals(bad):
    plan = np.zeros(4, dtype=np.int32)
    a = dict(m=100, n=100, k=128, dtype=rl.RLKV_BF16, plan=plan.ctypes.data)
    a.update(bad)
    assert rl.load_library().rlkv_plan_matmul(*a.values()) == -1
    assert (plan == 0).all()
    if "plan" not in bad:
        with pytest.raises(rl.RlkvError):
            rl.rlkv_plan_matmul(*list(a.values())[:4])
