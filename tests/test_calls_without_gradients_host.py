"""The calls on a caller's cache have no gradient: tensors that want one are refused, so that none is lost unsaid."""
import pytest
import torch

import paper_2511_18191_amd as tsd

APPEND = ("q", "k", "v", "k_pool", "v_pool", "page_table", "base", "freq")
ATTN = ("q", "k_pool", "v_pool", "page_table", "lens")


def some():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    i32 = torch.int32
    return dict(q=z(2, 3, 8, 64), k=z(2, 3, 4, 64), v=z(2, 3, 4, 64), k_pool=z(9, 16, 4, 64), v_pool=z(9, 16, 4, 64), page_table=z(2, 4, dtype=i32),
                base=z(2, dtype=i32), freq=z(32, dtype=torch.float64), lens=z(2, dtype=i32), out=z(2, 3, 8, 64))


@pytest.mark.parametrize("call,names,wants", [(tsd.rope_append_static, APPEND, n) for n in ("q", "k", "v", "k_pool", "v_pool", "freq", "out")]
                         + [(tsd.paged_attn_static, ATTN, n) for n in ("q", "k_pool", "v_pool", "out")])
def test_refused_while_gradients_are_recorded(call, names, wants):
    a = some()
    a[wants].requires_grad_()
    args = [a[n] for n in names]
    with pytest.raises(ValueError, match=f"{wants}.*gradient"):
        call(*args, out=a["out"])
    a[wants] = a[wants] * 2                    # no leaf: computed from one
    with pytest.raises(ValueError, match=f"{wants}.*gradient"):
        call(*[a[n] for n in names], out=a["out"])
    for mode in (torch.no_grad, torch.inference_mode):
        with mode(), pytest.raises(ValueError, match="cuda"):          # (the next check: these are the host's)
            call(*args, out=a["out"])


def test_probabilities_may_want_one():
    # what the verification returns are whole numbers, which have none in torch either
    p = torch.zeros(2, 4, 10, requires_grad=True)
    with pytest.raises(ValueError, match="cuda"):
        tsd.verify_tokens_static(torch.zeros(2, 3, dtype=torch.int64), p[:, :3], p, torch.zeros(2, 4))
