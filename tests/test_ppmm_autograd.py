"""The clear track and autograd (no GPU: the library is a stand-in that does nothing): no gradient is lost in silence, and a result
that autograd keeps for a backward pass is not overwritten in silence."""
import pytest
import torch

import paper_2601_18511_amd as pkg
from paper_2601_18511_amd import ppmm

T, M, K, D = 3, 4, 8, 64


class Library:
    def __getattr__(self, name):
        return lambda *args: 0


@pytest.fixture
def calls(monkeypatch):
    """{name: (call of the tensors, float inputs, outputs)} on CPU tensors."""
    monkeypatch.setattr(ppmm, "_lib", Library())
    monkeypatch.setattr(ppmm, "_handle", lambda device, stream: 0)
    plan = pkg.PpmvPlan(None, M, K, 32, torch.bfloat16, -1)
    plan.handle = 1
    cache = object.__new__(pkg.PpkvCache)
    cache.kv_heads, cache.head_dim, cache.device, cache._c = 1, D, -1, ppmm._CCache(0x1000, 1, 16, 1, D)
    where = torch.tensor([0, T], dtype=torch.int32), torch.tensor([T], dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32)
    rows = lambda w: torch.ones((T, w), dtype=torch.bfloat16)                     # noqa: E731
    heads = lambda: torch.ones((T, 1, D), dtype=torch.bfloat16)                   # noqa: E731
    yield {
        "ppmv_run": (lambda x, y: pkg.ppmv_run(plan, x, y), [rows(K)], [rows(M)]),
        "ppmv_gated_run": (lambda x, y: pkg.ppmv_gated_run(plan, plan, x, y), [rows(K)], [rows(M)]),
        "ppkv_append": (lambda k, v: pkg.ppkv_append(cache, k, v, *where), [heads(), heads()], []),
        "ppkv_read": (lambda k, v: pkg.ppkv_read(cache, k, v, *where), [], [heads(), heads()]),
        "ppkv_attention": (lambda q, o: pkg.ppkv_attention(cache, q, o, *where, max_q=T), [heads()], [heads()]),
    }
    plan.handle = None


NAMES = ("ppmv_run", "ppmv_gated_run", "ppkv_append", "ppkv_read", "ppkv_attention")


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_require_gradients(calls, name):
    call, inputs, outputs = calls[name]
    tensors = inputs + outputs
    call(*tensors)
    for t in tensors:
        t.requires_grad_(True)
        with pytest.raises(ValueError, match="no_grad"):
            call(*tensors)
        with torch.no_grad():
            call(*tensors)
        with torch.inference_mode():
            call(*tensors)
        t.requires_grad_(False)
        call(*tensors)


@pytest.mark.parametrize("name", NAMES)
def test_results_get_a_new_version(calls, name):
    call, inputs, outputs = calls[name]
    for grad in (True, False):
        with torch.set_grad_enabled(grad):
            before = [t._version for t in inputs + outputs]
            call(*inputs, *outputs)
            after = [t._version for t in inputs + outputs]
        assert after[:len(inputs)] == before[:len(inputs)]
        assert all(a > b for a, b in zip(after[len(inputs):], before[len(inputs):]))


def test_a_saved_result_that_is_overwritten_ends_the_backward_pass(calls):
    call, (x,), (y,) = calls["ppmv_run"]
    w = torch.ones((T, M), dtype=torch.bfloat16, requires_grad=True)
    call(x, y)
    loss = (w * y).sum()
    call(x, y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_one_result_of_a_read_may_be_unwanted(calls):
    call, _, (k, v) = calls["ppkv_read"]
    before = k._version
    call(k, None)
    call(None, v)
    assert k._version > before


def test_tensors_of_inference_mode(calls):
    with torch.inference_mode():
        for name in NAMES:
            call, inputs, outputs = calls[name]
            call(*[t.clone() for t in inputs + outputs])
