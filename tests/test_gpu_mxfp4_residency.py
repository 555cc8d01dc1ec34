"""GPU: decode batches over MXFP4 pages for each side of the rule that runs one workgroup a CU or two (equal items; neither
equal nor binned; binned and short; binned and more than three rounds of the CUs; long binned items of few rounds), with
the plan's facts that choose the side asserted."""
import numpy as np
import pytest

from tests.gpu_util import assert_attention_close
from tests.mxfp4_util import MxSetup, mx_case

pytestmark = pytest.mark.gpu

UNIFORM, BINNED, SORTED = 1, 2, 0
BATCHES = [  # long rows of a length, short rows of up to a length, the plan's order, more than 768 items, more than 2048 keys
    ("equal", 64, 512, 0, 0, UNIFORM, False, False),
    ("sorted", 8, 2500, 260, 60, SORTED, True, True),
    ("binned, short", 8, 700, 60, 300, BINNED, False, False),
    ("binned, many", 8, 2500, 92, 60, BINNED, True, True),
    ("binned, long, few", 8, 2500, 60, 60, BINNED, False, True),
    ("binned, pieces, few", 3, 9000, 24, 60, BINNED, False, True),
]


@pytest.mark.parametrize("what,long,length,short,most,order,many,far", BATCHES)
def test_decode_batches_on_each_side_of_the_rule(what, long, length, short, most, order, many, far):
    rng = np.random.default_rng(short)
    P = np.concatenate([np.full(long, length), rng.integers(1, max(most, 2), short)])
    rng.shuffle(P)
    case = mx_case("residency", P, [1] * len(P), 32, 8, seed=90)
    s = MxSetup(case)
    s.append()
    out, lse = s.attention()
    longest = min(P.max() + 1, s.plan.split_keys) if s.plan.split_keys else P.max() + 1
    assert (s.plan.tile_cols, s.plan.flags, s.plan.num_items > 3 * 256, longest > 2048) == (16, order, many, far)
    rows = {r: [0] for r in rng.choice(len(P), 16, replace=False).tolist() + [int(P.argmax()), int(P.argmin())]}
    assert_attention_close(case, out, lse, s.oracle(sample_rows=rows), rows, what=what)
