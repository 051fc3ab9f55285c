"""What the calls for a round of the caller's own models refuse of tensors, as Python's own errors, before anything is launched."""
import pytest
import torch

import paper_2511_18191_amd as tsd

pytestmark = pytest.mark.gpu


def some():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    i32 = torch.int32
    return dict(q=z(2, 3, 8, 64), k=z(2, 3, 4, 64), v=z(2, 3, 4, 64), k_pool=z(9, 16, 4, 64), v_pool=z(9, 16, 4, 64), page_table=z(2, 4, dtype=i32),
                base=z(2, dtype=i32), freq=z(32, dtype=torch.float64), lens=z(2, dtype=i32))


APPEND = ("q", "k", "v", "k_pool", "v_pool", "page_table", "base", "freq")
ATTN = ("q", "k_pool", "v_pool", "page_table", "lens")


@pytest.mark.parametrize("name,change", [
    ("q", lambda x: x.bfloat16()), ("q", lambda x: x[0]), ("q", lambda x: x.cpu()), ("q", lambda x: x[..., :32]), ("q", lambda x: x[..., ::2]),
    ("k", lambda x: x[:, :, :2]), ("k", lambda x: x.bfloat16()), ("v", lambda x: x[:, :2]), ("k_pool", lambda x: x.half()), ("k_pool", lambda x: x[0]),
    ("v_pool", lambda x: x[:5]), ("v_pool", lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)), ("v_pool", lambda x: x.cpu()),
    ("page_table", lambda x: x.long()), ("page_table", lambda x: x[:1]), ("page_table", lambda x: x.cpu()), ("page_table", lambda x: x[:, ::2]),
    ("page_table", lambda x: x[:1].expand(2, 4)), ("base", lambda x: x.long()), ("base", lambda x: x[:1]), ("base", lambda x: x.cpu()),
    ("freq", lambda x: x.float()), ("freq", lambda x: x[None]), ("freq", lambda x: x[::2]), ("lens", lambda x: x.long()), ("lens", lambda x: x.cpu()),
])
def test_tensors(name, change):
    for call, names in ((tsd.rope_append_static, APPEND), (tsd.paged_attn_static, ATTN)):
        if name in names:
            args = some()
            args[name] = change(args[name])
            with pytest.raises(ValueError):
                call(*[args[n] for n in names])


def test_options_and_outputs():
    a = some()
    append = lambda **o: tsd.rope_append_static(*[a[n] for n in APPEND], **o)
    attn = lambda **o: tsd.paged_attn_static(*[a[n] for n in ATTN], **o)
    i32 = torch.int32
    for call in (append, attn):
        for out in (a["q"].bfloat16(), a["q"][:1], a["q"][:1].expand(2, 3, 8, 64), a["q"].cpu()):
            with pytest.raises(ValueError):
                call(out=out)
        for n_new in (torch.zeros(3, dtype=i32).cuda(), torch.zeros(2).cuda(), torch.zeros(2, dtype=i32)):
            with pytest.raises(ValueError):
                call(n_new=n_new)
        with pytest.raises(TypeError):
            call(n_new=[1, 2])
    with pytest.raises(ValueError):
        append(positions=torch.zeros(2, 4, dtype=i32).cuda())
    with pytest.raises(TypeError):
        append(amplitude="1")
    with pytest.raises(tsd.TsdError, match="scale"):
        attn(scale=float("inf"))
    # what only the library knows to be wrong: rows off 16 bytes, heads that do not divide, an odd page size
    odd = torch.zeros(2 * 3 * 8 * 64 + 1, device="cuda")[1:].view(2, 3, 8, 64)
    with pytest.raises(tsd.TsdError, match="16 bytes"):
        tsd.paged_attn_static(odd, *[a[n] for n in ATTN[1:]])
    with pytest.raises(tsd.TsdError, match="multiple"):
        tsd.paged_attn_static(a["q"][:, :, :6], *[a[n] for n in ATTN[1:]])
    with pytest.raises(tsd.TsdError, match="page_tokens"):
        tsd.paged_attn_static(a["q"], a["k_pool"][:, :12], a["v_pool"][:, :12], a["page_table"], a["lens"])
    with pytest.raises(tsd.TsdError, match="B >= 1"):
        tsd.paged_attn_static(a["q"][:0], a["k_pool"], a["v_pool"], a["page_table"][:0], a["lens"][:0])


def test_drafts():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")
    draft, q, p, u = z(2, 3, dtype=torch.int64), z(2, 3, 50), z(2, 4, 50), z(2, 4)
    for args in ((draft.float(), q, p, u), (draft[0], q, p, u), (draft.cpu(), q, p, u), (draft[:, :2], q, p, u), (draft, q.bfloat16(), p, u), (draft, q[:, :2], p, u),
                 (draft, q[..., :49], p, u), (draft, q, p[:, :3], u), (draft, q, p.half(), u), (draft, q, p.transpose(1, 2), u), (draft, q, p, u[:, :3]),
                 (draft, q, p, u.double()), (draft, q, p, u.cpu()), (draft, q, p.cpu(), u)):
        with pytest.raises(ValueError):
            tsd.verify_tokens_static(*args)
    with pytest.raises(ValueError):
        tsd.verify_tokens_static(draft, q, p, u, n_draft=z(2))
    with pytest.raises(tsd.TsdError, match="16 drafts"):
        tsd.verify_tokens_static(z(2, 17, dtype=torch.int64), None, z(2, 18, 50), z(2, 18))
    with pytest.raises(tsd.TsdError, match="V >= 1"):
        tsd.verify_tokens_static(draft, q[..., :0], p[..., :0], u)
