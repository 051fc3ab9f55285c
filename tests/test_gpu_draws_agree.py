"""verify_tokens_static and verify_tree_static draw by one definition: the first token whose running sum passes u times the whole."""
import pytest
import torch

import paper_2511_18191_amd as tsd
from tree_ref import walked

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,V", [(40, 1), (40, 7), (30, 1000), (30, 1024), (20, 1025), (20, 5000), (10, 32000), (6, 50257), (3, 131072), (2, 300001)])
def test_the_chain_and_the_tree_draw_the_same(dtype, B, V):
    # Weights that are small whole numbers, most of them 0: sums in 64 bits are exact in every order.  Every u is a multiple of 1 / 64, so
    # that u W may meet a running sum exactly, or lies beside it by one unit of 32 bits.
    g = torch.Generator().manual_seed(V + B)
    p = (torch.randint(0, 4, (B, 1, V), generator=g) * (torch.rand(B, 1, V, generator=g) < 0.3)).float()
    u = torch.randint(0, 64, (B, 1), generator=g) / 64.0
    for b in range(0, B, 3):                                     # (u W is a whole number: W a multiple of 64)
        p[b, 0, V - 1] = 0.0
        p[b, 0, V - 1] = -float(p[b].double().sum()) % 64
    u[1::4] = torch.nextafter(u[1::4], torch.tensor(1.0))
    u[2::4] = torch.nextafter(u[2::4], torch.tensor(0.0)).clamp(min=0.0)
    p[B // 2] = 0.0                                              # nothing to draw
    p = p.to(dtype)
    zeros = torch.zeros(B, 1, dtype=torch.int32)
    tree = tsd.verify_tree_static(zeros.cuda(), zeros.cuda(), p=p.cuda(), uniforms=u.cuda())
    none = torch.zeros(B, dtype=torch.int32).cuda()
    chain = tsd.verify_tokens_static(zeros.cuda(), None, p.expand(B, 2, V).contiguous().cuda(), u.expand(B, 2).contiguous().cuda(), n_draft=none)
    _, want, _ = walked(zeros, zeros, p, u)
    assert tree["tokens"].tolist() == want
    assert chain["tokens"][:, :1].tolist() == want and not chain["n_acc"].any()
