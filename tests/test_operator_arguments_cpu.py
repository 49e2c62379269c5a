"""What the operators without a handle refuse, on the host alone: every check comes before the first CUDA call."""
import pytest
import torch

import __graft_entry__ as g

SOME = 1 << 20  # stands for a device address; nothing reads it


@pytest.fixture(scope="module")
def p():
    g.build()
    import paper_1810_09868_b200 as pkg
    return pkg


def logprobs_args(**over):
    a = dict(logits=SOME, dtype=1, rows=2, classes=10, ld=10, ids=SOME, n_ids=1, top_k=1, logprob=SOME, lse=SOME, entropy=SOME,
             top_id=SOME, top_logprob=SOME, stream=None)
    a.update(over)
    return tuple(a.values())


@pytest.mark.parametrize("over,code", [
    (dict(logits=None), "ARG"), (dict(dtype=2), "ARG"), (dict(rows=-1), "SHAPE"), (dict(rows=(1 << 26) + 1), "SHAPE"),
    (dict(classes=0, ld=0), "SHAPE"), (dict(classes=(1 << 30) + 1, ld=1 << 31), "SHAPE"), (dict(ld=9), "SHAPE"),
    (dict(n_ids=-1), "ARG"), (dict(n_ids=257), "ARG"), (dict(ids=None), "ARG"), (dict(logprob=None), "ARG"),
    (dict(top_k=-1), "ARG"), (dict(top_k=33), "ARG"), (dict(top_id=None), "ARG"), (dict(top_logprob=None), "ARG"),
    (dict(logits=SOME + 1), "ARG"), (dict(dtype=0, logits=SOME + 2), "ARG")])
def test_logprobs_refuses(p, over, code):
    assert p.binding.load().vgg19_logprobs(*logprobs_args(**over)) == getattr(p, "VGG19_ERR_" + code)
    assert p.vgg19_last_error()


def test_no_rows_is_no_work(p):
    lib = p.binding.load()
    assert lib.vgg19_logprobs(*logprobs_args(rows=0, logits=None, ids=None)) == p.VGG19_OK
    assert lib.vgg19_logprobs_backward(None, 0, 0, 5, 5, None, 0, None, None, None, None, None, 5, None) == p.VGG19_OK


@pytest.mark.parametrize("over,code", [
    (dict(lse=None), "ARG"), (dict(d_logits=None), "ARG"), (dict(d_logprob=None), "ARG"), (dict(entropy=None), "ARG"),
    (dict(d_ld=9), "SHAPE"), (dict(ld=9), "SHAPE"), (dict(d_logits=SOME + 1), "ARG"), (dict(n_ids=300), "ARG"),
    (dict(rows=1 << 26, classes=1 << 30, ld=1 << 30, d_ld=1 << 30), "SHAPE")])
def test_logprobs_backward_refuses(p, over, code):
    a = dict(logits=SOME, dtype=1, rows=2, classes=10, ld=10, ids=SOME, n_ids=1, lse=SOME, entropy=SOME, d_logprob=SOME,
             d_entropy=SOME, d_logits=SOME, d_ld=10, stream=None)
    a.update(over)
    assert p.binding.load().vgg19_logprobs_backward(*a.values()) == getattr(p, "VGG19_ERR_" + code)


def test_the_binding_refuses_host_tensors_and_wrong_types(p):
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_logprobs(torch.zeros(2, 5))
    assert e.value.code == p.VGG19_ERR_ARG
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_logprobs(torch.zeros(2, 5, dtype=torch.float64))
    assert e.value.code == p.VGG19_ERR_ARG
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_logprobs(torch.zeros(5))
    assert e.value.code == p.VGG19_ERR_SHAPE
