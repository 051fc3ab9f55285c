"""The extension of the calls on torch's tensors may be older than the package: what it holds goes on working, the rest says what to do."""
import sys
import types

import pytest

import paper_2511_18191_amd as tsd
from paper_2511_18191_amd import binding


@pytest.fixture
def older(monkeypatch):
    """An extension that knows the acceptance call only."""
    bound = []
    m = types.ModuleType("paper_2511_18191_amd._torch_calls")
    m.bind = bound.append
    m.accept_commit_static = lambda *a: (0, "n_acc", "commit", "ell", "logu")
    monkeypatch.setitem(sys.modules, m.__name__, m)
    monkeypatch.setattr(tsd, "_torch_calls", m, raising=False)
    for name in ("_calls", "_round_calls"):
        monkeypatch.setattr(binding, name, None, raising=False)
    return bound


def test_the_acceptance_call_needs_no_newer_extension(older):
    got = tsd.accept_commit_static(None, None, None, 0.5)
    assert got["n_acc"] == "n_acc" and len(older) == 1 and older[0]


@pytest.mark.parametrize("call", [
    lambda: tsd.rope_append_static(None, None, None, None, None, None, None, None),
    lambda: tsd.paged_attn_static(None, None, None, None, None),
    lambda: tsd.verify_tokens_static(None, None, None, None),
])
def test_the_calls_of_a_round_say_that_it_is_to_be_built(older, call):
    with pytest.raises(RuntimeError, match="_torch_calls.so.*build"):
        call()
    tsd.accept_commit_static(None, None, None, 0.5)
