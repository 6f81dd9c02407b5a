"""Every kernel and merge that the plan of ygg_tree_attention_block4 chooses, each against the definition on a small problem that takes it
(the plan is asserted, also without a GPU), and lengths far apart."""
import numpy as np
import pytest

import paper_2512_23858_amd as ygg
from test_gpu_block4 import _attend, _problem, _shape
from test_gpu_block8 import _check

# plan: row blocks, row blocks of the rest, several row tiles, cut into runs, twice the wavefronts, lanes to a row of the merge
PLANS = [  # B, Hq, Hkv, Dh, N, bound, plan
    (1, 8, 8, 128, 1, 130, (1, 0, False, False, False, 0)), (1, 8, 8, 128, 1, 300, (1, 0, False, False, True, 0)),
    (20, 32, 8, 128, 8, 4096, (1, 0, False, True, False, 16)), (1, 8, 8, 128, 1, 700, (1, 0, False, True, False, 64)),
    (1, 8, 1, 128, 5, 130, (2, 0, False, False, False, 0)), (16, 8, 8, 128, 33, 700, (2, 0, False, False, True, 0)),
    (3, 32, 32, 128, 49, 2000, (2, 0, False, True, False, 16)), (1, 8, 1, 128, 5, 700, (2, 0, False, True, False, 64)),
    (2, 32, 32, 128, 65, 130, (4, 0, False, False, False, 0)), (16, 8, 1, 128, 9, 300, (4, 0, False, False, True, 0)),
    (2, 32, 32, 128, 65, 700, (4, 0, False, True, False, 16)), (1, 8, 1, 128, 9, 300, (4, 0, False, True, False, 64)),
    (16, 64, 8, 128, 17, 130, (8, 0, False, False, False, 0)), (4, 64, 8, 128, 17, 130, (8, 0, False, True, False, 16)),
    (1, 8, 1, 128, 17, 130, (8, 0, False, True, False, 64)), (6, 64, 8, 128, 81, 130, (8, 0, True, False, False, 0)),
    (1, 64, 8, 128, 81, 130, (8, 0, True, True, False, 16)), (1, 8, 1, 128, 81, 130, (8, 0, True, True, False, 64)),
    (16, 64, 8, 128, 33, 130, (8, 2, False, False, False, 0)), (2, 64, 8, 128, 33, 130, (8, 2, False, True, False, 16)),
    (1, 8, 1, 128, 33, 130, (8, 2, False, True, False, 64)), (16, 32, 8, 128, 81, 130, (8, 4, False, False, False, 0)),
    (2, 32, 8, 128, 81, 130, (8, 4, False, True, False, 16)), (1, 32, 8, 128, 81, 130, (8, 4, False, True, False, 64)),
    (1, 8, 8, 64, 1, 130, (1, 0, False, False, False, 0)), (1, 8, 8, 64, 1, 300, (1, 0, False, False, True, 0)),
    (20, 32, 8, 64, 8, 4000, (1, 0, False, True, False, 8)), (1, 8, 8, 64, 1, 2000, (1, 0, False, True, False, 64)),
    (1, 8, 1, 64, 5, 130, (2, 0, False, False, False, 0)), (1, 8, 1, 64, 5, 300, (2, 0, False, False, True, 0)),
    (16, 8, 8, 64, 33, 2000, (2, 0, False, True, False, 8)), (1, 8, 1, 64, 5, 2000, (2, 0, False, True, False, 64)),
    (1, 8, 1, 64, 9, 130, (4, 0, False, False, False, 0)), (1, 8, 1, 64, 9, 300, (4, 0, False, False, True, 0)),
    (2, 32, 32, 64, 65, 700, (4, 0, False, True, False, 8)), (1, 8, 1, 64, 9, 700, (4, 0, False, True, False, 64)),
    (4, 32, 8, 64, 33, 130, (8, 0, False, False, False, 0)), (1, 32, 32, 64, 129, 0, (8, 0, False, True, False, 8)),
    (1, 8, 1, 64, 17, 300, (8, 0, False, True, False, 64)), (16, 8, 1, 64, 81, 130, (8, 0, True, False, False, 0)),
    (1, 64, 8, 64, 81, 130, (8, 0, True, True, False, 8)), (1, 8, 1, 64, 81, 130, (8, 0, True, True, False, 64)),
    (16, 8, 1, 64, 33, 130, (8, 2, False, False, False, 0)), (2, 64, 8, 64, 33, 130, (8, 2, False, True, False, 8)),
    (1, 8, 1, 64, 33, 130, (8, 2, False, True, False, 64)), (6, 32, 8, 64, 81, 130, (8, 4, False, False, False, 0)),
    (2, 32, 8, 64, 81, 130, (8, 4, False, True, False, 8)), (1, 32, 8, 64, 81, 130, (8, 4, False, True, False, 64)),
]


def _kind(shape):
    p = ygg.block4_plan(shape)
    return (p["row_blocks"], p["rem_blocks"], p["row_tiles"] > 1, p["runs"] > 1 or p["rem_runs"] > 1, p["wide"], p["merge_lanes"])


@pytest.mark.parametrize("B,Hq,Hkv,Dh,N,bound,plan", PLANS)
def test_plan_is_the_one_that_the_shape_is_here_for(B, Hq, Hkv, Dh, N, bound, plan):
    assert _kind(_shape(B, Hq, Hkv, Dh, N, bound + 1, most=bound)) == plan


def test_every_kind_of_plan_is_among_them():
    for Dh in (64, 128):
        kinds = {plan for *_, d, _, _, plan in PLANS if d == Dh}
        for B in (1, 2, 3, 6, 16, 40):
            for Hq, Hkv in ((8, 8), (32, 32), (40, 40), (32, 8), (64, 8), (8, 1), (12, 12), (2, 1)):
                for N in (1, 2, 5, 8, 9, 13, 17, 33, 49, 65, 81, 129, 145, 161, 257, 289, 321, 1024):
                    for bound in (0, 63, 130, 300, 700, 2000, 4096, 9000, 40000):
                        k = _kind(_shape(B, Hq, Hkv, Dh, N, bound + 1, most=bound))
                        # (the number of row tiles beside a rest makes no difference to the kernel)
                        assert any(k == o or (k[1] and k[:2] + k[3:] == o[:2] + o[3:]) for o in kinds), (B, Hq, Hkv, Dh, N, bound, k)


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,Dh,N,bound,plan", PLANS)
def test_attention_of_every_plan(B, Hq, Hkv, Dh, N, bound, plan):
    lens = np.random.default_rng(B + N + bound).integers(0, bound + 1, B)
    lens[0] = bound
    if B > 2:
        lens[1], lens[2] = 0, min(64, bound)
    p = _problem(B, Hq, Hkv, Dh, N, lens.tolist(), seed=N, cap=bound)
    assert _kind(p["shape"]) == plan
    _check(p, *_attend(p), sequences=sorted({0, 1 % B, B // 2, B - 1}))


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,Dh,N", [(8, 32, 32, 128, 49), (8, 32, 8, 128, 1), (12, 12, 12, 64, 17), (5, 40, 40, 128, 9)])
@pytest.mark.parametrize("bound", [1000, 4096])
def test_attention_one_long_sequence_among_short_ones(B, Hq, Hkv, Dh, N, bound):
    for lens in ([bound] + [70 + b for b in range(B - 1)], [0] * (B - 1) + [bound]):
        p = _problem(B, Hq, Hkv, Dh, N, lens, seed=N, cap=bound)
        _check(p, *_attend(p), sequences=[0, B // 2, B - 1])
