"""Dropout and the last layer with its loss where calls meet one another, and at the ends of what they take."""
import math

import pytest
import torch

import seeded_inputs as si

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


@pytest.mark.parametrize("graph", [True, False])
def test_a_pass_right_behind_set_dropout_takes_its_masks(p, graph):
    """On a stream that is not ordered behind the library's own copies: the masks, logits and gradients of a pass that waited for everything."""
    B = 3
    images, labels = torch.from_numpy(si.images(B, 32, 32, seed=1)).to(DEV).bfloat16(), torch.from_numpy(si.labels(B, seed=2)).to(DEV)
    net = p.Net(32, 32, B, p.VGG19_BF16, seed=1, flags=0 if graph else p.VGG19_FLAG_NO_GRAPH)
    logits = torch.empty(B, 1000, device=DEV)
    ones = torch.ones(B, 4096, device=DEV, dtype=torch.bfloat16)
    kept = torch.empty_like(ones)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for k in range(12):
            got = []
            for wait in (True, False):
                net.set_dropout(0.5, seed=7, first_pass=3)  # (another state in between)
                net.backward(images, labels, logits=logits)
                net.set_dropout(0.25, seed=100 + k, first_pass=5 * k)
                if wait:
                    torch.cuda.synchronize()
                for _ in range(2):  # the second pass counts on from the first
                    grads, _ = net.backward(images, labels, logits=logits)
                    got.append((logits.clone(), grads.clone()))
                act = net.saved_tensor(B, p.VGG19_MODE_BACKWARD, 21).reshape(B, -1)
                p.vgg19_dropout(ones, kept, 0.25, 100 + k, 2 * (5 * k + 1), stream=st)
                assert (act[kept == 0] == 0).all() and (act[kept != 0] != 0).any()
            for i in (0, 1):
                assert torch.equal(got[i][0], got[2 + i][0]) and torch.equal(got[i][1], got[2 + i][1])
            assert not torch.equal(got[0][0], got[1][0])
    net.sync_status(st)
    net.close()
