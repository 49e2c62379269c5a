"""The operators around the classifier together, as a program uses them: answer over 4-bit weights, score the answer, take the
gradient of a loss with an entropy term through the last dense layer, update that layer's weights; and a whole network trained with
the orthogonalised update and answering over the re-packed weights."""
import numpy as np
import pytest
import torch

import seeded_inputs as si

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


@pytest.mark.parametrize("stream_kind", ["current", "own", "recorded"])
def test_answer_score_train_update(p, stream_kind):
    rows, inner, classes, group = 9, 700, 1000, 64
    gen = torch.Generator(device=DEV).manual_seed(11)
    w = torch.randn(classes, inner, generator=gen, device=DEV) * (2.0 / inner) ** 0.5
    x = torch.randn(rows, inner, generator=gen, device=DEV).abs()
    bias = torch.randn(classes, generator=gen, device=DEV) * 0.1
    ids = torch.randint(0, classes, (rows, 2), generator=gen, device=DEV, dtype=torch.int32)
    ids[0, 1] = p.VGG19_NO_CLASS
    f32 = dict(dtype=torch.float32, device=DEV)
    codes = torch.empty(p.vgg19_q4_code_bytes(classes, inner), dtype=torch.uint8, device=DEV)
    scales = torch.empty(p.vgg19_q4_scale_bytes(classes, inner, group), dtype=torch.uint8, device=DEV)
    logits, d_logits = torch.empty(rows, classes, **f32), torch.empty(rows, classes, **f32)
    logprob, lse, entropy = torch.empty(rows, 2, **f32), torch.empty(rows, **f32), torch.empty(rows, **f32)
    top_id, top_lp = torch.empty(rows, 5, dtype=torch.int32, device=DEV), torch.empty(rows, 5, **f32)
    g = torch.full((rows, 2), -0.5 / rows, **f32)
    h = torch.full((rows,), -0.01 / rows, **f32)
    grad, momentum = torch.empty_like(w), torch.zeros_like(w)
    table = p.vgg19_muon_tensors([(w, None, grad, momentum)])
    ws = torch.empty(p.vgg19_muon_workspace_bytes(table), dtype=torch.uint8, device=DEV)
    w0 = w.clone()

    def step(st):
        p.vgg19_q4_pack(w, group, codes, scales, st)
        p.vgg19_q4_linear(x, codes, scales, classes, group, bias, False, logits, None, st)
        p.vgg19_logprobs(logits, ids, logprob, lse, entropy, top_id, top_lp, st)
        p.vgg19_logprobs_backward(logits, ids, lse, entropy, g, h, d_logits, st)
        torch.mm(d_logits.t(), x, out=grad)
        p.vgg19_muon_update(table, 0.05, 0.9, 0.01, 5, True, ws, st)

    if stream_kind == "current":
        step(torch.cuda.current_stream())
    else:
        st = torch.cuda.Stream()
        step(st), torch.cuda.synchronize()  # (first uses outside the capture)
        w.copy_(w0), momentum.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            if stream_kind == "own":
                step(st)
            else:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=st):
                    step(st)
                graph.replay()
    torch.cuda.synchronize()
    p.vgg19_ops_status(torch.cuda.current_stream())

    # the same in 64 bits, step by step
    w64, x64 = w0.double(), x.double()
    pad = -inner % group
    parts = torch.nn.functional.pad(w0, (0, pad)).view(classes, -1, group)
    sc = (parts.abs().amax(2, keepdim=True) / torch.tensor(7.0, device=DEV)).to(torch.bfloat16).float()
    q = torch.where(sc > 0, (parts / sc).round().clamp(-8, 7), torch.zeros_like(parts)) * sc
    wq = q.view(classes, -1)[:, :inner].double()
    z = x64 @ wq.T + bias.double()
    assert ((logits.double() - z).abs() <= 200 * U * (x64.abs() @ wq.abs().T + 1)).all()
    z = logits.double()  # from here on at the logits that were there
    lp = torch.log_softmax(z, 1)
    ent = -(lp.exp() * lp).sum(1)
    assert torch.equal(top_id.long(), torch.sort(z, stable=True, dim=1, descending=True).indices[:, :5])
    want = lp.gather(1, ids.clamp_min(0).long()).masked_fill(ids < 0, 0.0)
    assert ((logprob.double() - want).abs() <= 80 * U * (1 + want.abs())).all()
    gm = g.double().masked_fill(ids < 0, 0.0)
    one = torch.zeros_like(z).scatter_add_(1, ids.clamp_min(0).long(), gm)
    dz = one - lp.exp() * (gm.sum(1, keepdim=True) + h.double()[:, None] * (lp + ent[:, None]))
    size = one.abs() + lp.exp() * (gm.abs().sum(1, keepdim=True) + h.double().abs()[:, None] * (lp.abs() + ent[:, None]))
    assert ((d_logits.double() - dz).abs() <= 100 * U * size * (1 + lp.abs())).all()
    u = grad.double() * 1.9  # momentum was zero: M = G, U = G + 0.9 M
    m = u / u.norm()
    tall = m.shape[0] > m.shape[1]
    m = m.T if tall else m
    for _ in range(5):
        a = m @ m.T
        m = 3.4445 * m + (-4.7750 * a + 2.0315 * (a @ a)) @ m
    m = m.T if tall else m
    want = (1 - 0.05 * 0.01) * w64 - 0.05 * max(1.0, classes / inner) ** 0.5 * m
    # the orthogonalised part within 2^-13 of its size (its test has the reasons), the sum rounded
    assert float((w.double() - want).norm()) <= 0.05 * (classes / inner) ** 0.5 * float(m.norm()) * 2.0 ** -13 + 2 * U * float(want.norm())


def test_a_network_trains_and_answers(p):
    """Five updates on one batch: the parameters stay finite, the packed copies follow them, and what the network answers is what a
    network made from its parameters answers."""
    params = si.vgg19_params(32, 32, seed=0, bf16_exact=True)
    net = p.Net(32, 32, 4, p.VGG19_BF16, params=params, flags=p.VGG19_FLAG_DENSE_Q4)
    x = torch.from_numpy(si.images(4, 32, 32, seed=1, bf16_exact=True)).to(DEV).to(torch.bfloat16)
    y = torch.from_numpy(si.labels(4, seed=2)).to(DEV)
    momentum = torch.zeros(net.n_params, device=DEV)
    for _ in range(5):
        grads, loss = net.backward(x, y)
        net.muon_step(grads, momentum, 1e-3)
    net.sync_status()
    p.vgg19_ops_status(torch.cuda.current_stream())
    assert torch.isfinite(loss).all()
    now = np.empty(net.n_params, dtype=np.float32)
    p.vgg19_get_params(net.handle, now)
    assert np.isfinite(now).all() and not np.array_equal(now, params)
    ids, lp = net.classify(x, 5)
    again = p.Net(32, 32, 4, p.VGG19_BF16, params=now, flags=p.VGG19_FLAG_DENSE_Q4)
    ids2, lp2 = again.classify(x, 5)
    assert torch.equal(ids, ids2) and torch.equal(lp, lp2)
    net.close(), again.close()


def test_two_streams_at_once(p):
    """Calls of every operator on two streams that overlap, each with its own tensors, give what they give alone."""
    def build(seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        z = torch.randn(50, 30011, generator=gen, device=DEV)
        w = torch.randn(300, 900, generator=gen, device=DEV)
        s = dict(z=z, lse=torch.empty(50, device=DEV), ent=torch.empty(50, device=DEV), tid=torch.empty(50, 7, dtype=torch.int32, device=DEV),
                 tlp=torch.empty(50, 7, device=DEV), w=w, x=torch.randn(5, 900, generator=gen, device=DEV), y=torch.empty(5, 300, device=DEV),
                 codes=torch.empty(p.vgg19_q4_code_bytes(300, 900), dtype=torch.uint8, device=DEV),
                 scales=torch.empty(p.vgg19_q4_scale_bytes(300, 900, 32), dtype=torch.uint8, device=DEV),
                 grad=torch.randn(300, 900, generator=gen, device=DEV), m=torch.zeros(300, 900, device=DEV))
        s["table"] = p.vgg19_muon_tensors([(s["w"], None, s["grad"], s["m"])])
        s["ws"] = torch.empty(p.vgg19_muon_workspace_bytes(s["table"]), dtype=torch.uint8, device=DEV)
        return s

    def run(s, st):
        p.vgg19_logprobs(s["z"], None, None, s["lse"], s["ent"], s["tid"], s["tlp"], st)
        p.vgg19_q4_pack(s["w"], 32, s["codes"], s["scales"], st)
        p.vgg19_q4_linear(s["x"], s["codes"], s["scales"], 300, 32, None, True, s["y"], None, st)
        p.vgg19_muon_update(s["table"], 0.1, 0.9, 0.0, 5, True, s["ws"], st)

    alone = [build(i) for i in (1, 2)]
    for s in alone:
        run(s, torch.cuda.current_stream())
        torch.cuda.synchronize()
    both = [build(i) for i in (1, 2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, st in zip(both, streams):
        run(s, st)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        for k in ("lse", "ent", "tid", "tlp", "codes", "scales", "y", "w", "m"):
            assert torch.equal(a[k], b[k]), k


def test_a_network_on_a_stream_given_by_its_address(p):
    net = p.Net(32, 32, 2, p.VGG19_BF16, seed=1, mode=p.VGG19_MODE_BACKWARD)
    images = torch.rand(2, 32, 32, 3, device=DEV).to(torch.bfloat16)
    grads, momentum = torch.full((net.n_params,), 1e-3, device=DEV), torch.zeros(net.n_params, device=DEV)
    before = net.classify(images)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    ids, logprob = net.classify(images, stream=st.cuda_stream)
    st.synchronize()
    assert torch.equal(ids, before[0]) and torch.equal(logprob, before[1])
    net.muon_step(grads, momentum, 0.01, stream=st.cuda_stream)
    st.synchronize()
    assert not torch.equal(net.classify(images)[1], logprob)
    net.close()


class _Unanswered:
    """Stands for the compiled calls, answering none of them."""

    def __getattr__(self, name):
        return lambda *a: None


def test_the_binding_without_its_compiled_calls_gives_the_same(p, monkeypatch):
    gen = torch.Generator(device=DEV).manual_seed(2)
    z = torch.randn(5, 700, generator=gen, device=DEV)[:, :603]
    ids = torch.randint(0, 603, (5, 2), generator=gen, device=DEV, dtype=torch.int32)
    codes = torch.randint(0, 256, (p.vgg19_q4_code_bytes(33, 603),), generator=gen, dtype=torch.uint8, device=DEV)
    scales = torch.rand(p.vgg19_q4_scale_bytes(33, 603, 64) // 2, generator=gen, device=DEV).to(torch.bfloat16)
    g, w, bias = torch.randn(5, 2, generator=gen, device=DEV), torch.randn(5, generator=gen, device=DEV), torch.randn(33, generator=gen, device=DEV)

    def all_calls(stream):
        o = dict(logprob=torch.empty(5, 2, device=DEV), lse=torch.empty(5, device=DEV), entropy=torch.empty(5, device=DEV),
                 top_id=torch.empty(5, 4, dtype=torch.int32, device=DEV), top_logprob=torch.empty(5, 4, device=DEV))
        d, y, yf = torch.empty(5, 603, device=DEV), torch.empty(5, 33, device=DEV), torch.empty(5, 33, device=DEV)
        assert p.vgg19_logprobs(z, ids, stream=stream, **o) == p.VGG19_OK
        assert p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, d, stream) == p.VGG19_OK
        assert p.vgg19_q4_linear(z, codes, scales, 33, 64, bias, True, y, yf, stream) == p.VGG19_OK
        torch.cuda.synchronize()
        return [*o.values(), d, y, yf]

    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = [all_calls(s) for s in (torch.cuda.current_stream(), st, st.cuda_stream, None)]
    monkeypatch.setattr(p.binding, "_tensor_calls", _Unanswered())
    for other in want[1:] + [all_calls(st), all_calls(st.cuda_stream), all_calls(None)]:
        for a, b in zip(want[0], other):
            assert torch.equal(a, b)


def test_two_host_threads(p):
    """Each with its own stream, buffers and refusals; what they get is what one alone gets."""
    import threading

    def job(seed, stream, out):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        rows, n = 40 + seed, 900 + 300 * seed
        with torch.cuda.stream(stream):
            z = torch.randn(rows, n, generator=gen, device=DEV)
            lse, top = torch.empty(rows, device=DEV), (torch.empty(rows, 6, dtype=torch.int32, device=DEV), torch.empty(rows, 6, device=DEV))
            codes = torch.randint(0, 256, (p.vgg19_q4_code_bytes(100 * seed, n),), generator=gen, dtype=torch.uint8, device=DEV)
            scales = torch.rand(p.vgg19_q4_scale_bytes(100 * seed, n, 64) // 2, generator=gen, device=DEV).to(torch.bfloat16)
            y = torch.empty(rows, 100 * seed, device=DEV)
            w, g, m = (torch.randn(70 * seed, 210, generator=gen, device=DEV) for _ in range(3))
            table = p.vgg19_muon_tensors([(w, None, g, m)])
            ws = torch.empty(p.vgg19_muon_workspace_bytes(table), dtype=torch.uint8, device=DEV)
            for _ in range(20):
                p.vgg19_logprobs(z, lse=lse, top_id=top[0], top_logprob=top[1], stream=stream)
                p.vgg19_q4_linear(z, codes, scales, 100 * seed, 64, y=y, stream=stream)
                p.vgg19_muon_update(table, 0.01, 0.9, 0.0, 5, True, ws, stream=stream)
                try:
                    p.vgg19_q4_linear(z, codes, scales, 100 * seed, 64, y=z, stream=stream)
                except p.Vgg19Error as e:
                    out.append(str(e))
            stream.synchronize()
        out += [lse, *top, y, w, m]

    alone, together = [[], []], [[], []]
    for i in range(2):
        job(i + 1, torch.cuda.Stream(), alone[i])
    torch.cuda.synchronize()
    threads = [threading.Thread(target=job, args=(i + 1, torch.cuda.Stream(), together[i])) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert len(a) == len(b) == 26 and a[:20] == b[:20]
        for x, y in zip(a[20:], b[20:]):
            assert torch.equal(x, y)
    p.vgg19_ops_status(torch.cuda.current_stream())
