"""Log probabilities, entropy, top alternatives and their gradient against plain arithmetic in 64 bits.

Tolerances.  With u = 2^-24 (half a step of fp32): a term exp(z - ref) carries the rounding of (z - ref) log2 e, which is
|z - ref| 1.5 u relative to the term, and 4 u of the exponential (its documented 2 ulp); terms far below the reference hardly
count, so 16 u covers a sum's terms.  Adding n of them in fp32 along chains of at most n / 128 + 32 (a lane's share of a row
that belongs to at least four warps, the joins after it) adds (n / 128 + 32) u.  Hence a relative error of (n / 128 + 48) u
for S = sum exp, the same absolute error for log S, and the rounding of what is stored.  The entropy is a sum of terms
p |log p|, off by as much relative to log S + H."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


def outputs(rows, n_ids, top):
    f = dict(dtype=torch.float32, device=DEV)
    nan = float("nan")
    return dict(logprob=torch.full((rows, n_ids), nan, **f), lse=torch.full((rows,), nan, **f), entropy=torch.full((rows,), nan, **f),
                top_id=torch.full((rows, top), -7, dtype=torch.int32, device=DEV), top_logprob=torch.full((rows, top), nan, **f))


def call(p, z, ids, top, stream=None):
    o = outputs(z.shape[0], ids.shape[1], top)
    p.vgg19_logprobs(z, ids, stream=stream or torch.cuda.current_stream(), **o)
    return o


def reference(z, ids, top):
    z = z.double().cpu()
    ids = ids.long().cpu()
    top_z = z.amax(1)
    empty = top_z == -math.inf
    rest = z - top_z[:, None]                  # subtracted first: at 3e38 even 64 bits would lose log S beside it
    logs = rest.exp().sum(1).log()
    lse = top_z + logs
    logp = rest - logs[:, None]
    logp[logp < -3.4028235e38] = -math.inf     # what fp32 holds
    lse[empty] = -math.inf
    logp[empty] = -math.inf
    pr = logp.exp()
    h = -torch.where(pr > 0, pr * logp, torch.zeros_like(pr)).sum(1)
    pad = ids < 0
    given = logp.gather(1, ids.clamp_min(0)).masked_fill(pad, 0.0)
    order = torch.sort(z, stable=True, dim=1, descending=True)
    k = min(top, z.shape[1])
    top_id = torch.full((z.shape[0], top), -1)
    top_lp = torch.full((z.shape[0], top), -math.inf, dtype=torch.float64)
    top_id[:, :k] = order.indices[:, :k]
    top_lp[:, :k] = logp.gather(1, order.indices[:, :k])
    top_id[:, :k][order.values[:, :k] == -math.inf] = -1  # excluded, which a finite logit never is
    return dict(logprob=given, lse=lse, entropy=h, top_id=top_id, top_logprob=top_lp), logp


def close(got, want, tol):
    got, want = got.double().cpu(), want.double().cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    return bool((same | ((got - want).abs() <= tol)).all())


def check(o, want, n):
    c = n / 128 + 48
    assert torch.equal(o["top_id"].cpu().long(), want["top_id"])
    fin = lambda t: torch.nan_to_num(t.abs(), posinf=0.0)  # noqa: E731
    assert close(o["lse"], want["lse"], (c + fin(want["lse"])) * U)
    for k in ("logprob", "top_logprob"):
        assert close(o[k], want[k], (c + 3 * fin(want[k])) * U), k
    assert close(o["entropy"], want["entropy"], 2 * c * U * (1 + math.log(max(n, 2)) + want["entropy"]))


def make(rows, n, dtype, seed=0, std=2.5, ld=None, offset=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ld = ld or n
    buf = torch.full((offset + rows * ld + 64,), float("nan"), dtype=TYPES[dtype], device=DEV)  # what lies between rows is never read
    z = buf[offset:offset + rows * ld].view(rows, ld)[:, :n]
    z.copy_(torch.randn(rows, n, generator=gen, device=DEV) * std)
    ids = torch.randint(0, n, (rows, 3), generator=gen, device=DEV, dtype=torch.int32)
    return z, ids


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(1, 1, 5), (3, 2, 1), (2, 5, 5), (1, 31, 32), (7, 32, 8), (5, 33, 32), (2, 127, 3), (100, 1000, 5),
                                        (1, 1000, 5), (4, 1025, 20), (1, 4096, 32), (9, 4097, 7), (1, 8191, 1), (2, 50021, 20),
                                        (1, 131072, 20), (300, 5003, 0), (40, 20011, 32)])
def test_rows(p, rows, n, top, dtype):
    z, ids = make(rows, n, dtype, seed=rows * n)
    ids[0, 0] = p.VGG19_NO_CLASS
    want, _ = reference(z, ids, top)
    check(call(p, z, ids, top), want, n)
    p.vgg19_ops_status(torch.cuda.current_stream())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("ld,offset", [(1009, 0), (1000, 1), (1003, 3), (1024, 7), (2001, 5)])
def test_strides_and_starts(p, ld, offset, dtype):
    z, ids = make(6, 1000, dtype, seed=ld, ld=ld, offset=offset)
    want, _ = reference(z, ids, 5)
    check(call(p, z, ids, 5), want, 1000)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [40, 3001, 70001])
def test_ties_go_to_the_lower_index(p, n, dtype):
    gen = torch.Generator(device=DEV).manual_seed(n)
    z = torch.randint(-3, 3, (4, n), generator=gen, device=DEV).to(TYPES[dtype])
    z[1] = 0.0
    z[1, ::2] = -0.0  # equal to 0
    z[2] = 1.5
    ids = torch.zeros(4, 1, dtype=torch.int32, device=DEV)
    want, _ = reference(z, ids, 32)
    check(call(p, z, ids, 32), want, n)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [500, 60000])
def test_sorted_rows(p, n, dtype):
    up = torch.linspace(-90, 90, n, device=DEV).to(TYPES[dtype])
    z = torch.stack([up, up.flip(0), torch.cat([up[::2], up[1::2]])])
    ids = torch.tensor([[0], [n - 1], [n // 2]], dtype=torch.int32, device=DEV)
    want, _ = reference(z, ids, 16)
    check(call(p, z, ids, 16), want, n)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n", [9, 1000, 40000])
def test_excluded_classes_and_extreme_values(p, n, dtype):
    z, ids = make(9, n, dtype, seed=n)
    low = torch.finfo(TYPES[dtype]).min
    z[0, 1:] = -math.inf             # one class left
    z[1] = -math.inf                 # none
    z[2, : n // 2] = low             # masks of the type's lowest value
    z[3] = low                       # nothing else
    z[4] = -low                      # all at the largest
    z[5, ::2], z[5, 1::2] = low, -low
    z[6, 3:] = -math.inf
    z[7] -= 1000
    z[8, n - 1] = 80.0               # nearly all of the mass
    want, _ = reference(z, ids, 6)
    check(call(p, z, ids, 6), want, n)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("at", [0, 17, 999])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_nan_or_infinity_shows_in_its_row_alone(p, at, value, dtype):
    z, ids = make(3, 1000, dtype)
    ids[1, 0] = p.VGG19_NO_CLASS
    clean = call(p, z, ids, 4)
    z[1, at] = value
    o = call(p, z, ids, 4)
    for k in ("lse", "entropy", "top_logprob"):
        assert torch.isnan(o[k][1]).all()
    assert o["logprob"][1, 0] == 0 and torch.isnan(o["logprob"][1, 1:]).all() and (o["top_id"][1] == p.VGG19_NO_CLASS).all()
    for k in o:
        assert torch.equal(o[k][0::2], clean[k][0::2])
    z[1] = -math.inf
    z[1, at] = math.nan
    assert torch.isnan(call(p, z, ids, 4)["lse"][1])


def test_ids_outside_the_classes(p):
    z, ids = make(4, 50, "fp32")
    ids[1, 1], ids[2, 0] = 50, -2
    o = call(p, z, ids, 2)
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_ops_status(torch.cuda.current_stream())
    assert e.value.code == p.VGG19_ERR_ARG
    p.vgg19_ops_status(torch.cuda.current_stream())  # reported once
    bad = torch.zeros(4, 3, dtype=torch.bool)
    bad[1, 1] = bad[2, 0] = True
    assert torch.equal(torch.isnan(o["logprob"]).cpu(), bad)
    # in the gradient they contribute nothing
    g = torch.ones(4, 3, device=DEV)
    d, d2 = torch.empty_like(z), torch.empty_like(z)
    p.vgg19_logprobs_backward(z, ids, o["lse"], None, g, None, d, torch.cuda.current_stream())
    with pytest.raises(p.Vgg19Error):
        p.vgg19_ops_status(torch.cuda.current_stream())
    ids[1, 1] = ids[2, 0] = p.VGG19_NO_CLASS
    p.vgg19_logprobs_backward(z, ids, o["lse"], None, g, None, d2, torch.cuda.current_stream())
    assert torch.equal(d, d2)


def test_parts_may_be_left_out(p):
    z, ids = make(5, 700, "bf16")
    full = call(p, z, ids, 3)
    st = torch.cuda.current_stream()
    o = outputs(5, 3, 3)
    p.vgg19_logprobs(z, lse=o["lse"], stream=st)
    p.vgg19_logprobs(z, ids, o["logprob"], stream=st)
    p.vgg19_logprobs(z, top_id=o["top_id"], top_logprob=o["top_logprob"], stream=st)
    for k in ("lse", "logprob", "top_id", "top_logprob"):
        assert torch.equal(o[k], full[k])
    empty = z[:0]
    p.vgg19_logprobs(empty, ids[:0], o["logprob"][:0], stream=st)
    p.vgg19_logprobs_backward(empty, None, o["lse"][:0], None, None, None, empty, st)


# ---- the gradient ------------------------------------------------------------------------------------------------

def upstream(rows, k, seed=5):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(rows, k, generator=gen, device=DEV), torch.randn(rows, generator=gen, device=DEV)


def check_gradient(d, z, ids, logp, h, lse, g, w):
    pr = logp.exp()
    ids, g, w = ids.long().cpu(), g.double().cpu(), w.double().cpu()
    pad = ids < 0
    g = g.masked_fill(pad, 0.0)
    alive = ~torch.isinf(lse)
    one = torch.zeros_like(logp).scatter_add_(1, ids.clamp_min(0), g) * alive[:, None]
    lp = torch.where(pr > 0, logp, torch.zeros_like(logp))
    want = one - pr * (g.sum(1, keepdim=True) + w[:, None] * (lp + h[:, None]))
    # p carries the rounding of lse and of (z - lse), the bracket a few roundings of its terms, the sums of d their own
    size = pr * (g.abs().sum(1, keepdim=True) + w.abs()[:, None] * (lp.abs() + h[:, None]))
    fin = torch.nan_to_num(lse.abs(), posinf=0.0)[:, None]
    tol = U * size * (3 * lp.abs() + 2 * fin + 32) + 4 * U * one.abs() + 2.0 ** -126 * (1 + size)
    if d.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    assert close(d, want, tol)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n,ld,d_ld,offset", [(1, 1, 1, 1, 0), (3, 7, 7, 7, 0), (5, 33, 40, 33, 1), (100, 1000, 1000, 1000, 0),
                                                   (4, 1025, 1025, 1025, 3), (2, 16385, 16385, 16390, 0), (1, 50021, 50021, 50021, 0)])
def test_gradient(p, rows, n, ld, d_ld, offset, dtype):
    z, ids = make(rows, n, dtype, seed=n, ld=ld, offset=offset)
    ids[0, 0] = p.VGG19_NO_CLASS
    if rows > 1:
        ids[1, 2] = ids[1, 0]            # the same class twice
    if rows > 2:
        z[2] = -math.inf                 # nothing left
    if n > 20:
        z[0, 5:15] = -math.inf
        z[0, 15] = torch.finfo(z.dtype).min
        ids[0, 1] = 7                    # an excluded class
    want, logp = reference(z, ids, 1)
    lse, h = want["lse"].float().to(DEV), want["entropy"].float().to(DEV)
    g, w = upstream(rows, 3)
    buf = torch.full((rows * d_ld,), 123.0, dtype=z.dtype, device=DEV)
    d = buf.view(rows, d_ld)[:, :n]
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, d, torch.cuda.current_stream())
    check_gradient(d, z, ids, logp, want["entropy"], want["lse"], g, w)
    assert (buf.view(rows, d_ld)[:, n:] == 123.0).all()  # what lies between the rows stays
    # without an entropy term, without ids
    zero = torch.zeros_like(w)
    p.vgg19_logprobs_backward(z, ids, lse, None, g, None, d, torch.cuda.current_stream())
    check_gradient(d, z, ids, logp, want["entropy"], want["lse"], g, zero)
    p.vgg19_logprobs_backward(z, None, lse, h, None, w, d, torch.cuda.current_stream())
    check_gradient(d, z, ids, logp, want["entropy"], want["lse"], torch.zeros_like(g), w)


@pytest.mark.parametrize("n_ids", [1, 40, 256])
def test_many_ids_and_repeats(p, n_ids):
    n = 9001
    z, _ = make(3, n, "fp32")
    gen = torch.Generator(device=DEV).manual_seed(n_ids)
    ids = torch.randint(0, 60, (3, n_ids), generator=gen, device=DEV, dtype=torch.int32)
    ids[:, n_ids // 2:] += n - 60
    want, logp = reference(z, ids, 1)
    o = call(p, z, ids, 1)
    check(o, want, n)
    g, w = upstream(3, n_ids)
    d, again = torch.empty_like(z), torch.empty_like(z)
    lse, h = want["lse"].float().to(DEV), want["entropy"].float().to(DEV)
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, d, torch.cuda.current_stream())
    # the sum over n_ids shares: n_ids more roundings of their total size
    ids64, g64 = ids.long().cpu(), g.double().cpu()
    slack = n_ids * U * (g64.abs().sum(1, keepdim=True) * logp.exp() + torch.zeros_like(logp).scatter_add_(1, ids64, g64.abs()))
    one = torch.zeros_like(logp).scatter_add_(1, ids64, g64)
    pr = logp.exp()
    exact = one - pr * (g64.sum(1, keepdim=True) + w.double().cpu()[:, None] * (logp + want["entropy"][:, None]))
    size = pr * (g64.abs().sum(1, keepdim=True) + w.double().cpu().abs()[:, None] * (logp.abs() + want["entropy"][:, None]))
    assert close(d, exact, slack + U * size * (3 * logp.abs() + 2 * want["lse"].abs()[:, None] + 32) + 4 * U * one.abs())
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, again, torch.cuda.current_stream())
    assert torch.equal(d, again)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_in_place(p, dtype):
    z, ids = make(7, 5001, dtype, ld=5003, offset=1)
    g, w = upstream(7, 3)
    o = call(p, z, ids, 1)
    d = torch.empty(7, 5001, dtype=z.dtype, device=DEV)
    p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, d, torch.cuda.current_stream())
    p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, z, torch.cuda.current_stream())
    assert torch.equal(z, d)


def test_gradient_against_differences(p):
    """Central differences of the forward kernel: step 2^-6; the third derivative of g log p + w H is below 10 (|g|, |w| < 3 here,
    probabilities sum to one), so h^2 / 6 times it, and the roundings of two fp32 results of size 10 over 2 h."""
    n, step = 11, 2.0 ** -6
    z, ids = make(1, n, "fp32", std=1.0)
    g, w = upstream(1, 3)
    o = call(p, z, ids, 1)
    d = torch.empty_like(z)
    p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, d, torch.cuda.current_stream())
    both = torch.cat([z + step * torch.eye(n, device=DEV), z - step * torch.eye(n, device=DEV)])
    o = call(p, both, ids.expand(2 * n, 3).contiguous(), 1)
    f = (o["logprob"].double() * g.double()).sum(1) + o["entropy"].double() * w.double()
    diff = (f[:n] - f[n:]) / (2 * step)
    assert (d[0].double() - diff).abs().max() <= 10 * step ** 2 / 6 * 3 + 64 * U * 10 / step


# ---- how it is called --------------------------------------------------------------------------------------------

def test_another_stream_and_a_recorded_graph(p):
    z, ids = make(64, 3001, "bf16")
    g, w = upstream(64, 3)
    o, d = outputs(64, 3, 5), torch.empty_like(z)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        p.vgg19_logprobs(z, ids, stream=st, **o)
        p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, d, st)
    for seed in (1, 2):
        z.copy_(make(64, 3001, "bf16", seed=seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        again = call(p, z, ids, 5)
        for k in o:
            assert torch.equal(o[k], again[k])
        d2 = torch.empty_like(z)
        p.vgg19_logprobs_backward(z, ids, again["lse"], again["entropy"], g, w, d2, torch.cuda.current_stream())
        assert torch.equal(d, d2)


def test_rows_beyond_32_bits(p):
    """The second row starts 2^31 elements after the first."""
    n = 1001
    buf = torch.empty((1 << 31) + n, dtype=torch.bfloat16, device=DEV)
    z = buf.as_strided((2, n), (1 << 31, 1))
    src, ids = make(2, n, "bf16", seed=3)
    z.copy_(src)
    want, logp = reference(src, ids, 4)
    o = call(p, z, ids, 4)
    check(o, want, n)
    g, w = upstream(2, 3)
    p.vgg19_logprobs_backward(z, ids, want["lse"].float().to(DEV), want["entropy"].float().to(DEV), g, w, z, torch.cuda.current_stream())
    check_gradient(z, src, ids, logp, want["entropy"], want["lse"], g, w)


def test_refusals(p):
    z, ids = make(4, 50, "fp32")
    o = outputs(4, 3, 2)
    st = torch.cuda.current_stream()

    def refused(code, **over):
        a = dict(o, logits=z, ids=ids, stream=st)
        a.update(over)
        with pytest.raises(p.Vgg19Error) as e:
            p.vgg19_logprobs(**a)
        assert e.value.code == code

    refused(p.VGG19_ERR_ARG, logits=z.half())
    refused(p.VGG19_ERR_ARG, logits=z.t().contiguous().t())
    refused(p.VGG19_ERR_ARG, logits=z[:1].expand(4, 50))
    refused(p.VGG19_ERR_ARG, ids=ids.long())
    refused(p.VGG19_ERR_ARG, ids=ids.cpu())
    refused(p.VGG19_ERR_SHAPE, ids=ids[:3])
    refused(p.VGG19_ERR_SHAPE, lse=o["lse"][:2])
    refused(p.VGG19_ERR_ARG, logprob=None)
    refused(p.VGG19_ERR_ARG, top_id=torch.zeros(4, 33, dtype=torch.int32, device=DEV), top_logprob=torch.zeros(4, 33, device=DEV))
    with pytest.raises(p.Vgg19Error):
        p.vgg19_logprobs_backward(z, ids, o["lse"], None, o["logprob"], o["entropy"], torch.empty_like(z), st)
    with pytest.raises(p.Vgg19Error):
        p.vgg19_logprobs_backward(z, ids, o["lse"], None, o["logprob"], None, torch.empty(4, 50, dtype=torch.bfloat16, device=DEV), st)


def test_the_network_names_its_best_classes(p):
    """Net.classify: the forward pass's logits through the same kernel."""
    import numpy as np
    import seeded_inputs as si
    net = p.Net(32, 32, 3, p.VGG19_BF16, params=si.vgg19_params(32, 32, seed=0, bf16_exact=True), mode=p.VGG19_MODE_FORWARD)
    x = torch.from_numpy(si.images(3, 32, 32, seed=1, bf16_exact=True)).to(DEV).to(torch.bfloat16)
    ids, lp = net.classify(x, 5)
    logits = net.forward(x)
    want, _ = reference(logits, torch.zeros(3, 1, dtype=torch.int32), 5)
    assert np.array_equal(ids.cpu().numpy(), want["top_id"].numpy())
    assert close(lp, want["top_logprob"], (1000 / 128 + 48 + 3 * want["top_logprob"].abs()) * U)
    net.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradient_beside_the_logits(p, dtype):
    """Logits and their gradient as the two halves of the same rows: nothing overlaps."""
    n = 1003
    src, ids = make(9, n, dtype, seed=4)
    both = torch.full((9, 2 * n + 1), float("nan"), dtype=src.dtype, device=DEV)
    z, beside = both[:, 1:n + 1], both[:, n + 1:]
    z.copy_(src)
    g, w = upstream(9, 3)
    o = call(p, z, ids, 1)
    d = torch.empty(9, n, dtype=z.dtype, device=DEV)
    p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, d, torch.cuda.current_stream())
    p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, beside, torch.cuda.current_stream())
    assert torch.equal(beside, d) and torch.equal(z, src) and torch.isnan(both[:, 0]).all()
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_logprobs_backward(z, ids, o["lse"], o["entropy"], g, w, both[:, :n], torch.cuda.current_stream())
    assert e.value.code == p.VGG19_ERR_ARG


# Rows that belong to one warp (see the kernels): a lane adds n / 32 terms, five joins follow; n / 32 + 5 <= n / 128 + 32 up to 1024.

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(1, 1, 1), (601, 3, 2), (5, 32, 32), (130, 33, 7), (2, 64, 32), (600, 65, 32), (3, 255, 9), (40, 256, 32),
                                        (2, 257, 32), (700, 512, 32), (6, 513, 8), (6, 513, 9), (513, 1000, 3), (7, 1023, 0), (600, 1024, 8), (3, 1024, 32),
                                        (2, 1025, 8)])
def test_short_rows(p, rows, n, top, dtype):
    z, ids = make(rows, n, dtype, seed=rows + n, ld=n + rows % 3, offset=n % 5)
    if rows > 2:
        z[1] = -math.inf                                   # nothing left
        z[2, : n // 2] = torch.finfo(z.dtype).min
        z[rows - 1, ::3] = z[rows - 1, 0].clone()          # ties
        ids[0, 1] = p.VGG19_NO_CLASS
    want, logp = reference(z, ids, top)
    o = call(p, z, ids, top)
    check(o, want, n)
    g, w = upstream(rows, 3)
    d = torch.empty(rows, n, dtype=z.dtype, device=DEV)
    lse, h = want["lse"].float().to(DEV), want["entropy"].float().to(DEV)
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, d, torch.cuda.current_stream())
    check_gradient(d, z, ids, logp, want["entropy"], want["lse"], g, w)
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, z, torch.cuda.current_stream())  # in place
    assert torch.equal(z, d)


@pytest.mark.parametrize("n", [20, 300, 800])
@pytest.mark.parametrize("n_ids", [33, 256])
def test_short_rows_many_ids(p, n, n_ids):
    rows = 512
    z, _ = make(rows, n, "fp32", seed=n)
    gen = torch.Generator(device=DEV).manual_seed(n_ids)
    ids = torch.randint(0, n, (rows, n_ids), generator=gen, device=DEV, dtype=torch.int32)
    ids[:, 5] = ids[:, 40 % n_ids]
    want, logp = reference(z, ids, 1)
    check(call(p, z, ids, 1), want, n)
    g, w = upstream(rows, n_ids)
    d, again = torch.empty_like(z), torch.empty_like(z)
    lse, h = want["lse"].float().to(DEV), want["entropy"].float().to(DEV)
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, d, torch.cuda.current_stream())
    ids64, g64, w64 = ids.long().cpu(), g.double().cpu(), w.double().cpu()[:, None]
    pr, h64 = logp.exp(), want["entropy"][:, None]
    given, shares = torch.zeros_like(logp).scatter_add_(1, ids64, g64), torch.zeros_like(logp).scatter_add_(1, ids64, g64.abs())
    exact = given - pr * (g64.sum(1, keepdim=True) + w64 * (logp + h64))
    size = pr * (g64.abs().sum(1, keepdim=True) + w64.abs() * (logp.abs() + h64))
    # as above: the sum over n_ids shares is n_ids more roundings of their total size
    slack = n_ids * U * (g64.abs().sum(1, keepdim=True) * pr + shares)
    assert close(d, exact, slack + U * size * (3 * logp.abs() + 2 * want["lse"].abs()[:, None] + 32) + 4 * U * given.abs())
    p.vgg19_logprobs_backward(z, ids, lse, h, g, w, again, torch.cuda.current_stream())
    assert torch.equal(d, again)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,at", [(7, 6), (64, 40), (250, 249), (500, 3), (1000, 500)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_short_rows_with_a_nan_or_infinity(p, n, at, value, dtype):
    z, ids = make(6, n, dtype)
    clean = call(p, z, ids, 4)
    z[3, at] = value
    o = call(p, z, ids, 4)
    for k in ("lse", "entropy", "top_logprob", "logprob"):
        assert torch.isnan(o[k][3]).all()
        assert torch.equal(o[k][:3], clean[k][:3]) and torch.equal(o[k][4:], clean[k][4:])
    assert (o["top_id"][3] == p.VGG19_NO_CLASS).all()
    bad = ids.clone()
    bad[0, 0], bad[4, 2] = n, -2
    o = call(p, z, bad, 4)
    assert torch.isnan(o["logprob"][0, 0]) and torch.isnan(o["logprob"][4, 2]) and torch.equal(o["logprob"][1:3], clean["logprob"][1:3])
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_ops_status(torch.cuda.current_stream())
    assert e.value.code == p.VGG19_ERR_ARG
    g, w = upstream(6, 3)
    d = torch.empty_like(z)
    p.vgg19_logprobs_backward(z, bad, o["lse"], o["entropy"], g, w, d, torch.cuda.current_stream())
    assert torch.isnan(d[3]).all() and not torch.isnan(d[:3]).any() and not torch.isnan(d[4:]).any()
    with pytest.raises(p.Vgg19Error):
        p.vgg19_ops_status(torch.cuda.current_stream())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n,top", [(3, 2000, 1), (2, 9001, 32), (1, 131072, 20), (300, 50021, 3)])
def test_rows_of_equals(p, rows, n, top, dtype):
    """What a classifier answers before it has learnt anything; and a few classes that stand out of equals, below and above."""
    z = torch.zeros(rows, n, dtype=TYPES[dtype], device=DEV)
    if rows > 1:
        z[1, 5::7] = -1.0
        z[1, n - 3:] = 2.0
        z[rows - 1] = torch.linspace(-4, 4, n, device=DEV).to(TYPES[dtype])  # bf16: runs of equals
    ids = torch.zeros(rows, 1, dtype=torch.int32, device=DEV)
    want, _ = reference(z, ids, top)
    check(call(p, z, ids, top), want, n)
