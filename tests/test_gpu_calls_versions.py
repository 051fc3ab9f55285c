"""Tensors that the calls on a caller's cache write count as changed in place: autograd does not go on with what it saved of them."""
import pytest
import torch

import paper_2511_18191_amd as tsd

pytestmark = pytest.mark.gpu


def some():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    i32 = torch.int32
    return dict(q=z(2, 3, 8, 64), k=z(2, 3, 4, 64), v=z(2, 3, 4, 64), k_pool=z(9, 16, 4, 64), v_pool=z(9, 16, 4, 64),
                page_table=torch.arange(8, dtype=i32, device="cuda").view(2, 4), base=z(2, dtype=i32), freq=z(32, dtype=torch.float64),
                lens=torch.full((2,), 3, dtype=i32, device="cuda"), out=z(2, 3, 8, 64))


def append(a, **o):
    return tsd.rope_append_static(*[a[n] for n in ("q", "k", "v", "k_pool", "v_pool", "page_table", "base", "freq")], **o)


def attn(a, **o):
    return tsd.paged_attn_static(*[a[n] for n in ("q", "k_pool", "v_pool", "page_table", "lens")], **o)


def versions(a):
    return {n: t._version for n, t in a.items()}


def changed(before, a):
    return {n for n, t in a.items() if t._version != before[n]}


def test_versions():
    a = some()
    before = versions(a)
    append(a, out=a["out"])
    assert changed(before, a) == {"k_pool", "v_pool", "out"}
    before = versions(a)
    append(a)
    assert changed(before, a) == {"k_pool", "v_pool"}
    before = versions(a)
    attn(a, out=a["out"])
    assert changed(before, a) == {"out"}
    before = versions(a)
    attn(a, out=a["q"])
    assert changed(before, a) == {"q"}
    before = versions(a)
    with pytest.raises(tsd.TsdError):
        attn(a, out=a["out"], scale=float("inf"))
    assert changed(before, a) == set()


def test_a_saved_tensor_that_a_call_wrote_is_noticed():
    a, w = some(), torch.ones(9, 16, 4, 64, device="cuda", requires_grad=True)
    y = (w * a["k_pool"]).sum()                # saves the pool for w's gradient
    with torch.no_grad():
        append(a)
    with pytest.raises(RuntimeError, match="inplace|in-place"):
        y.backward()


def test_tensors_of_inference_mode():
    # they have no versions: written all the same, inside that mode and outside
    with torch.inference_mode():
        a = some()
        a["q"] += 1.0
        a["v"] += 2.0
        append(a, out=a["out"])
        assert bool((a["v_pool"][0, :3] == 2.0).all()) and bool((attn(a) == 2.0).all())
    a["out"][0].cpu()
    append(a, out=a["out"])
    assert bool((attn(a, out=a["out"]) == 2.0).all())
