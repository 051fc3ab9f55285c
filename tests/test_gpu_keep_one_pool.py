"""keep_path_static where a model's keys are its values: one pool under both names, moved once."""
import pytest
import torch

import paper_2511_18191_amd as tsd
from test_gpu_keep_path import BF, FP, inputs
from tree_ref import kept

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,N,L,cols,page,H,D", [(2, 40, 1, 4, 16, 1, 64), (3, 256, 2, 20, 16, 3, 128), (40, 64, 3, 6, 16, 8, 128), (1, 200, 5, 300, 1, 1, 256)])
def test_keys_that_are_values(dtype, B, N, L, cols, page, H, D):
    pool, _, table, held, path = inputs(B, N, L, cols, page, H, D, dtype)
    path[0] = torch.arange(0, 2 * N, 2).where(torch.arange(N) < N // 2, torch.tensor(-1))     # (every row's source is an earlier row's place)
    want = kept(pool.cpu(), table, held, path, page)
    tsd.keep_path_static(pool, pool, table.cuda(), held.cuda(), path.cuda())
    assert torch.equal(pool.cpu(), want)
