"""What the calls for rounds of trees, windowed caches and scores refuse of tensors, as Python's own errors, before anything is launched."""
import pytest
import torch

import paper_2511_18191_amd as tsd

pytestmark = pytest.mark.gpu
i32 = torch.int32


def z(*s, dtype=torch.float32):
    return torch.zeros(*s, dtype=dtype, device="cuda")


def refused(call, *changes):
    for change in changes:
        with pytest.raises(ValueError):
            call(**change)


def attn(call):
    a = dict(q=z(2, 3, 8, 64), k_pool=z(9, 16, 4, 64), v_pool=z(9, 16, 4, 64), page_table=z(2, 4, dtype=i32), lens=z(2, dtype=i32))
    return a, lambda **o: call(**{**a, **o})


def test_window():
    a, call = attn(lambda **o: tsd.window_attn_static(o.pop("q"), o.pop("k_pool"), o.pop("v_pool"), o.pop("page_table"), o.pop("lens"), o.pop("window", 7), **o))
    assert call().shape == a["q"].shape
    q, k, t = a["q"], a["k_pool"], a["page_table"]
    refused(call, dict(q=q.bfloat16()), dict(q=q[0]), dict(q=q.cpu()), dict(q=q[..., :32]), dict(q=q[..., ::2]), dict(k_pool=k.half()), dict(v_pool=k[:5]),
            dict(page_table=t.long()), dict(page_table=t[:1]), dict(page_table=t[:1].expand(2, 4)), dict(lens=z(2)), dict(lens=z(3, dtype=i32)), dict(n_new=z(2)),
            dict(n_new=z(3, dtype=i32)), dict(out=q.bfloat16()), dict(out=q[:1].expand(2, 3, 8, 64)), dict(window=2 ** 40), dict(sinks=-2 ** 40))
    for o in (dict(window=0), dict(window=-5), dict(sinks=-1), dict(scale=float("inf"))):
        with pytest.raises(tsd.TsdError):
            call(**o)
    for o in (dict(window=2.5), dict(window=None), dict(sinks="1"), dict(n_new=[1, 2])):
        with pytest.raises(TypeError):
            call(**o)


def test_tree():
    a, call = attn(lambda **o: tsd.tree_attn_static(o.pop("q"), o.pop("k_pool"), o.pop("v_pool"), o.pop("page_table"), o.pop("lens"),
                                                    o.pop("parents", z(2, 3, dtype=i32)), **o))
    assert call().shape == call(parents=z(3, dtype=i32)).shape == a["q"].shape
    refused(call, *[dict(parents=x) for x in (z(2, 3), z(2, 3, dtype=torch.int64), z(2, 4, dtype=i32), z(1, 3, dtype=i32), z(2, dtype=i32), z(2, 3, dtype=i32).cpu(),
                                              z(3, 2, dtype=i32).t(), z(1, 3, dtype=i32).expand(2, 3))],
            dict(q=a["q"].bfloat16()), dict(lens=z(2)), dict(window=0), dict(window=-1))
    with pytest.raises(TypeError):
        call(parents=[-1, 0, 1])
    with pytest.raises(tsd.TsdError, match="256"):
        call(q=z(2, 257, 8, 64), parents=z(257, dtype=i32))


def test_scores():
    logits, tokens = z(2, 3, 50), z(2, 3, dtype=torch.int64)
    call = lambda **o: tsd.token_logprobs_static(o.pop("logits", logits), **{"tokens": tokens, **o})
    assert set(call(top=2)) == {"logprobs", "entropy", "top_ids", "top_logprobs"}
    refused(call, *[dict(logits=x) for x in (logits.half(), logits.double(), logits[0], logits.cpu(), logits[..., ::2], logits.transpose(1, 2))],
            *[dict(tokens=x) for x in (tokens.float(), tokens[0], tokens.cpu(), tokens[:, :2], tokens.t().contiguous().t())],
            dict(n_new=z(2)), dict(n_new=z(3, dtype=i32)), dict(top=-1))
    for o in (dict(top=33), dict(temperature=0.0), dict(temperature=float("nan")), dict(logits=logits[..., :0])):
        with pytest.raises(tsd.TsdError):
            call(**o)
    for o in (dict(tokens=[[1]]), dict(top="3"), dict(temperature="1"), dict(top=1.5)):
        with pytest.raises(TypeError):
            call(**o)


def test_walks():
    a = dict(tokens=z(2, 5, dtype=i32), parents=z(2, 5, dtype=i32), p=z(2, 5, 50), uniforms=z(2, 5))
    call = lambda **o: tsd.verify_tree_static(**{**a, **o})
    assert set(call()) == {"n_acc", "tokens", "path"}
    refused(call, *[dict(tokens=x) for x in (a["tokens"].float(), a["tokens"][0], a["tokens"].cpu(), a["tokens"][:, :4], a["tokens"].t().contiguous().t())],
            *[dict(parents=x) for x in (a["parents"].long(), a["parents"][:1], a["parents"].cpu(), z(2, dtype=i32))],
            *[dict(p=x) for x in (a["p"].half(), a["p"].cpu(), a["p"][:, :4], a["p"].transpose(1, 2), None)],
            *[dict(uniforms=x) for x in (z(2, 4), z(2, 5).double(), z(2, 5).cpu(), None)], dict(n_new=z(2)), dict(choices=z(2, 5, dtype=i32)),
            dict(p=None, uniforms=None), dict(p=None, uniforms=None, choices=z(2, 5, dtype=torch.int64)), dict(p=None, choices=z(2, 5, dtype=i32)))
    with pytest.raises(tsd.TsdError, match="256"):
        tsd.verify_tree_static(z(1, 257, dtype=i32), z(257, dtype=i32), p=z(1, 257, 2), uniforms=z(1, 257))
    with pytest.raises(tsd.TsdError, match="V >= 1"):
        call(p=a["p"][..., :0])
    with pytest.raises(TypeError):
        call(tokens=[[1]])


def test_kept_paths():
    k = z(3, 9, 16, 4, 64)
    a = dict(k_pool=k, v_pool=z(3, 9, 16, 4, 64), page_table=z(2, 4, dtype=i32), held=z(2, dtype=i32), path=z(2, 5, dtype=i32))
    call = lambda **o: tsd.keep_path_static(**{**a, **o})
    call()
    refused(call, *[dict(k_pool=x) for x in (k[0], k.bfloat16(), k.cpu(), k[:2], k[:1].expand(3, 9, 16, 4, 64), k[:0])], dict(v_pool=k.transpose(2, 3)),
            dict(page_table=a["page_table"].long()), dict(held=z(2)), dict(held=z(3, dtype=i32)), dict(path=z(2, 5)), dict(path=z(3, 5, dtype=i32)),
            dict(path=z(5, 2, dtype=i32).t()), dict(path=z(5, dtype=i32)), dict(path=a["path"].cpu()),
            dict(k_pool=k[0, :1].expand(9, 16, 4, 64), v_pool=k[0, :1].expand(9, 16, 4, 64)))
    with pytest.raises(tsd.TsdError, match="256"):
        call(path=z(2, 257, dtype=i32))
