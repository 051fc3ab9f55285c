"""token_logprobs_static where logits and temperatures are as large as their types hold, against its definition in 64 bits (tests/tree_ref.py)."""
import pytest
import torch

import paper_2511_18191_amd as tsd
from tree_ref import check_scores, scores

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,V", [(3, 2), (3, 100), (2, 5000), (520, 300), (1, 100000)])
@pytest.mark.parametrize("temperature", [1e-6, 1.0, 1e30, 1e38, 3.4e38])
def test_logits_and_temperatures_of_any_size(dtype, B, V, temperature):
    # differences of logits pass the type's largest number, and a factor of 1 / 3.4e38 its least normal one; what is left after both is ordinary
    g = torch.Generator().manual_seed(V)
    logits = ((2 * torch.rand(B, 1, V, generator=g, dtype=torch.float64) - 1) * torch.finfo(dtype).max).to(dtype).cuda()
    logits[0, 0, 0], logits[0, 0, V - 1] = -torch.finfo(dtype).max, torch.finfo(dtype).max
    tokens = torch.randint(0, V, (B, 1), generator=g).cuda()
    tokens[0] = 0
    for top in (0, 7):
        got = tsd.token_logprobs_static(logits, tokens, top=top, temperature=temperature)
        check_scores(got, *scores(logits, tokens, top, temperature))
