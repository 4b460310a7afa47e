"""What lies in key blocks that no list names has no influence, whatever it is, also on lists with an odd number of units."""
import math

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import sequence_oracle as orc
from sequence_util import f64, normal
from test_gpu_sequence_attention import bounds, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("N,share,picked", [
    (3, 2, [0, 4, 5]),              # 6 rows
    (9, 3, [0, 4, 5]),              # 27
    (30, 2, [1]),                   # 60
    (50, 2, [0, 4, 5]),             # 100
    (50, 2, [3]),
    (100, 8, [7, 2, 0, 4, 5]),      # 800
])
def test_blocks_that_are_not_listed(what, dtype, d, N, share, picked):
    M, block = 300, 32                  # (the newest block, which every row sees in part, is not listed)
    Q, dO = (normal((1, share, N, d), dtype, 400 + i) for i in range(2))
    K, V = (normal((1, 1, M, d), dtype, 402 + i) for i in range(2))
    index = np.full((1, 1, 1, 6), -1, np.int32)
    index[..., :len(picked)] = picked
    count = np.full((1, 1, 1), len(picked), np.int32)
    mask = orc.attended(count, index, N, M, N, block, True)
    for j in range(-(-M // block)):
        if j not in picked:
            K[:, :, j * block:(j + 1) * block] = what
            V[:, :, j * block:(j + 1) * block] = what
    scale = 1 / math.sqrt(d)
    lists = torch.from_numpy(count).cuda(), torch.from_numpy(index).cuda()
    O, lse = grat.grat_selected_attention_fwd(Q, K, V, scale, *lists, q_group=N, block=block, return_lse=True)
    grads = grat.grat_selected_attention_bwd(dO, Q, K, V, O, lse, scale, *lists, q_group=N, block=block)
    Ow, _, bO, _, want, lims = bounds(*(f64(t) for t in (Q, K, V)), scale, mask, dtype, f64(dO))
    within(f64(O), Ow, bO, "O")
    for name, got, w, lim in zip(("dQ", "dK", "dV"), grads, want, lims):
        within(f64(got), w, lim, name)
