"""What trains a classifier's head, together: features of a network, dropout, the last layer with its loss, the gradients back, an update; and dropout
inside a network's own training passes."""
import math

import numpy as np
import pytest
import torch

import seeded_inputs as si
from test_gpu_dropout import expected

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


class Head:
    """A head of many classes on the features of a network's second dense layer."""

    def __init__(self, p, features, labels, classes, dtype):
        g = torch.Generator(device=DEV).manual_seed(2)
        self.p, self.labels = p, labels
        self.x = features.to(dtype)
        rows, inner = self.x.shape
        self.w32 = torch.randn(classes, inner, generator=g, device=DEV) / math.sqrt(inner)
        self.w, self.bias = self.w32.to(dtype), torch.zeros(classes, device=DEV)
        self.y, self.dy, self.dx = (torch.empty_like(self.x) for _ in range(3))
        self.dw, self.db = torch.empty_like(self.w32), torch.empty(classes, device=DEV)
        self.loss, self.lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        self.momentum = torch.zeros_like(self.w32)
        self.d_loss = torch.full((rows,), 1.0 / rows, device=DEV)
        self.counter = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.ws = [torch.empty(p.vgg19_linear_cross_entropy_bytes(self.x, self.w, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
        self.table = p.vgg19_muon_tensors([(self.w32, self.w if dtype == torch.bfloat16 else None, self.dw, self.momentum)])
        self.update_ws = torch.empty(p.vgg19_muon_workspace_bytes(self.table), dtype=torch.uint8, device=DEV)

    def gradients(self, st):
        p = self.p
        p.vgg19_dropout(self.x, self.y, 0.5, 3, 0, self.counter, stream=st)
        p.vgg19_linear_cross_entropy(self.y, self.w, self.bias, self.labels, self.loss, self.lse, self.ws[0], st)
        p.vgg19_linear_cross_entropy_backward(self.y, self.w, self.bias, self.labels, self.lse, self.d_loss, self.dy, self.dw, self.db, self.ws[1], st)
        p.vgg19_dropout_backward(self.dy, self.dx, 0.5, 3, 0, self.counter, stream=st)

    def step(self, st):
        self.gradients(st)
        self.p.vgg19_muon_update(self.table, 0.02, 0.9, 0.0, 5, True, self.update_ws, stream=st)
        self.bias.sub_(self.db, alpha=0.02)
        self.counter.add_(1)


def features(p, batch):
    net = p.Net(32, 32, batch, p.VGG19_BF16, seed=0, mode=p.VGG19_MODE_FORWARD)
    images = torch.from_numpy(si.images(batch, 32, 32, seed=1)).to(DEV).bfloat16()
    net.forward(images)
    f = net.saved_tensor(batch, p.VGG19_MODE_FORWARD, 22).clone().view(batch, 4096)
    net.sync_status()
    net.close()
    return f / f.float().std().item()


@pytest.mark.parametrize("dtype,half", [(torch.bfloat16, 2.0 ** -8), (torch.float32, 2.0 ** -24)])
def test_gradients_through_the_head(p, dtype, half):
    """Against autograd in 64 bits over the same mask, in the 2-norm: bf16 rounds y, dz and the result, dx once more, each at most by h relative; fp32 sums are
    within 1e-5 of theirs."""
    batch, classes = 20, 5003
    labels = torch.from_numpy(si.labels(batch, seed=3)).to(DEV).int()
    h = Head(p, features(p, batch), labels, classes, dtype)
    h.gradients(torch.cuda.current_stream())
    p.vgg19_ops_status(torch.cuda.current_stream())
    mask = expected(torch.ones(batch, 4096, device=DEV), 0.5, 3).double()
    x, w, b = h.x.double().requires_grad_(), h.w.double().requires_grad_(), h.bias.double().requires_grad_()
    y = x * mask
    y = y + (y.to(dtype).double() - y).detach()  # (y is stored in its type)
    loss = torch.nn.functional.cross_entropy(y @ w.T + b, labels.long(), reduction="none")
    (loss.mean()).backward()
    near = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert near(h.loss, loss.detach()) < 1e-5
    assert near(h.dw, w.grad) < 2 * half + 1e-5 and near(h.db, b.grad) < 2e-5 and near(h.dx, x.grad) < 4 * half + 1e-5


def test_training_steps_recorded_and_one_by_one(p):
    """Steps of a bf16 head, called and replayed: the same bits, and a loss of its own mask each time."""
    batch, classes = 20, 1000
    labels = torch.from_numpy(si.labels(batch, seed=3)).to(DEV).int()
    f = features(p, batch)
    eager, recorded = (Head(p, f, labels, classes, torch.bfloat16) for _ in range(2))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        losses = []
        for _ in range(4):
            eager.step(st)
            losses.append(eager.loss.clone())
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        recorded.step(torch.cuda.current_stream())
    for k in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(recorded.loss, losses[k])
    for n in ("w32", "w", "bias", "momentum", "dx", "counter"):
        assert torch.equal(getattr(eager, n), getattr(recorded, n)), n
    assert len({float(v.sum()) for v in losses}) == 4
    p.vgg19_ops_status(st)


def network_pass(p, net, images, labels, params):
    """One backward pass; (activations behind dense 1 and 2, logits, gradients)."""
    logits = torch.empty(len(images), 1000, device=DEV)
    grads, _ = net.backward(images, labels, logits=logits)
    net.sync_status()
    act = [net.saved_tensor(len(images), p.VGG19_MODE_BACKWARD, i).reshape(len(images), -1).float().clone() for i in (20, 21, 22)]
    return act, logits, grads.clone()


@pytest.mark.parametrize("graph", [True, False])
def test_dropout_in_a_networks_training_passes(p, graph):
    """fp32 at 32 x 32: the dense layers in 64 bits over the masks of the pass's steps, from the features that the pass stored."""
    B = 3
    params = si.vgg19_params(32, 32, seed=0)
    images, labels = torch.from_numpy(si.images(B, 32, 32, seed=1)).to(DEV), torch.from_numpy(si.labels(B, seed=2)).to(DEV)
    net = p.Net(32, 32, B, p.VGG19_FP32, params=params, flags=0 if graph else p.VGG19_FLAG_NO_GRAPH)
    slices = net.param_slices()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()

    def at(flat, i):
        off, dims = slices[i]
        return flat[off:off + int(np.prod(dims))].reshape(dims)

    with torch.cuda.stream(st):
        plain = network_pass(p, net, images, labels, params)
        net.set_dropout(0.5, seed=77, first_pass=4)
        for step in (8, 10, 12):
            (f, a1, a2), logits, grads = network_pass(p, net, images, labels, params)
            assert torch.equal(f, plain[0][0])
            ones = torch.ones(B, 4096, device=DEV)
            m = [expected(ones, 0.5, 77, step + k).double() for k in range(2)]
            w = [torch.from_numpy(np.ascontiguousarray(at(params, i))).to(DEV).double().requires_grad_() for i in range(32, 38)]
            h1 = torch.relu(f.double() @ w[0].T + w[1]) * m[0]
            h2 = torch.relu(h1 @ w[2].T + w[3]) * m[1]
            z = h2 @ w[4].T + w[5]
            torch.nn.functional.cross_entropy(z, labels.long()).backward()
            for got, want in [(a1, h1.detach()), (a2, h2.detach()), (logits, z.detach())] + [(at(grads, 32 + i), w[i].grad) for i in range(6)]:
                assert float((got.double() - want).norm() / want.norm()) < 1e-5
            assert not torch.equal(grads[:slices[32][0]], plain[2][:slices[32][0]])  # the convolutions' gradients pass through the masks
        net.set_dropout(0.0)
        again = network_pass(p, net, images, labels, params)
        assert torch.equal(again[1], plain[1]) and torch.equal(again[2], plain[2])
        logits = net.forward(images).clone()
        net.set_dropout(0.5)
        assert torch.equal(net.forward(images), logits)  # answers have none
    net.close()


def test_training_programs_count_passes(p):
    """Three steps as one program, three recorded steps and passes that start at a later step: the same parameters."""
    B, lr = 2, 1e-3
    images = torch.from_numpy(si.images(B * 3, 32, 32, seed=1)).to(DEV).bfloat16()
    labels = torch.from_numpy(si.labels(B * 3, seed=2)).to(DEV)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()

    def network():
        net = p.Net(32, 32, B, p.VGG19_BF16, seed=1, mode=p.VGG19_MODE_TRAIN)
        net.set_dropout(0.3, seed=5)
        return net

    def parameters(net):
        out = np.empty(net.n_params, dtype=np.float32)
        st.synchronize()
        p.vgg19_get_params(net.handle, out)
        net.sync_status(st)
        net.close()
        return out

    with torch.cuda.stream(st):
        a, b, c = network(), network(), network()
        p.vgg19_train_steps(a.handle, images, labels, B, 3, lr, None, st)
        x, y = images[:B].clone(), labels[:B].clone()
        for k in range(3):
            x.copy_(images[B * k:B * k + B]), y.copy_(labels[B * k:B * k + B])
            b.train_step(x, y, lr, stream=st)
            c.set_dropout(0.3, seed=5, first_pass=k)
            c.train_step(x, y, lr, stream=st)
        got = [parameters(n) for n in (a, b, c)]
    assert np.array_equal(got[0], got[1]) and np.array_equal(got[0], got[2])


def test_a_layers_wait_that_runs_out_is_reported_once(p):
    st = torch.cuda.current_stream()
    p.vgg19_ops_status(st)
    ws = torch.empty(p.VGG19_SELFTEST_BYTES, dtype=torch.uint8, device=DEV)
    p.vgg19_selftest_operator_timeout(None, p.VGG19_SELFTEST_LOSS, ws, st)
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_ops_status(st)
    assert e.value.code == p.VGG19_ERR_DEVICE_TIMEOUT and "loss" in str(e.value)
    p.vgg19_ops_status(st)
    net = p.Net(32, 32, 1, p.VGG19_BF16, seed=1, mode=p.VGG19_MODE_FORWARD)
    p.vgg19_selftest_operator_timeout(net.handle, p.VGG19_SELFTEST_LOSS, ws, st)
    p.vgg19_ops_status(st)
    with pytest.raises(p.Vgg19Error) as e:
        net.sync_status()
    assert e.value.code == p.VGG19_ERR_DEVICE_TIMEOUT
    net.sync_status()
    net.close()
    labels = torch.zeros(20, dtype=torch.int32, device=DEV)  # and the operator works as it did
    h = Head(p, torch.randn(20, 4096, device=DEV), labels, 1000, torch.bfloat16)
    h.gradients(st)
    p.vgg19_ops_status(st)
    z = h.y.double() @ h.w.double().T
    assert float((h.loss.double() - (torch.logsumexp(z, 1) - z[:, 0])).abs().max()) < 1e-4
