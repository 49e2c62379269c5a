"""The orthogonalised update against the same iteration in 64 bits.

Tolerances.  One step maps singular values by f(s) = a s + b s^3 + c s^5; on [0, 1.21], where they stay, |f'| <= 4.3, so an error
of X in the Frobenius norm grows by at most that factor a step (the matrix function's derivative has the divided differences of f as
its entries).  Operands hold 22 bits (2^-22 relative to their size), a step multiplies three times and every product's sums add about
as much again: 8 * 2^-22 of |X|_F a step, |X|_F <= 1.21 sqrt(m).  The early errors count most, and |X_0|_F = 1: the sum over the steps
stays below  GROW^steps * 8 * 2^-22 * (1 + sqrt(m) / 8)  for the sizes here.  That is a worst case; test_as_close_as_fp32 holds typical
matrices to the error of the plain fp32 iteration (24 bits) times four, the ratio of the operands' steps."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
A, B, C = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


def gradient(rows, cols, seed, rank=None, std=1e-2):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    g = torch.randn(rows, cols, generator=gen, device=DEV) * std
    if rank:
        g = g * 0.01 + torch.randn(rows, rank, generator=gen, device=DEV) @ torch.randn(rank, cols, generator=gen, device=DEV) * std
    return g


def tensors(rows, cols, seed=0, rank=None, offset=0, w16=True):
    gen = torch.Generator(device=DEV).manual_seed(seed + 1000)
    n = rows * cols

    def place(v, dt=torch.float32):
        buf = torch.full((n + offset + 8,), 77.0, dtype=dt, device=DEV)
        out = buf[offset:offset + n].view(rows, cols)
        out.copy_(v)
        return out

    w = torch.randn(rows, cols, generator=gen, device=DEV) * 0.1
    m = torch.randn(rows, cols, generator=gen, device=DEV) * 1e-3
    return (place(w), place(w, torch.bfloat16) if w16 else None, place(gradient(rows, cols, seed, rank)), place(m))


def iterate(x, steps, dt=torch.float64):
    x = x.to(dt)
    for _ in range(steps):
        a = x @ x.T
        x = A * x + (B * a + C * (a @ a)) @ x
    return x


def reference(t, lr, mu, decay, steps, nesterov, dt=torch.float64):
    w, _, g, m = (None if v is None else v.to(dt) for v in t)
    m = mu * m + g
    u = g + mu * m if nesterov else m
    x = u / u.double().norm().to(dt)
    rows, cols = x.shape
    x = iterate(x, steps, dt) if rows <= cols else iterate(x.T, steps, dt).T
    return (1 - lr * decay) * w - lr * math.sqrt(max(1.0, rows / cols)) * x, m, x


def run(p, ts, lr=0.02, mu=0.95, decay=0.01, steps=5, nesterov=True, stream=None, fill=0xff):
    table = p.vgg19_muon_tensors(ts)
    ws = torch.full((p.vgg19_muon_workspace_bytes(table),), fill, dtype=torch.uint8, device=DEV)  # NaN in every format
    p.vgg19_muon_update(table, lr, mu, decay, steps, nesterov, ws, stream=stream or torch.cuda.current_stream())
    p.vgg19_ops_status(stream or torch.cuda.current_stream())


def check(t, before, lr, mu, decay, steps, nesterov):
    want, m, x = reference(before, lr, mu, decay, steps, nesterov)
    rows, cols = x.shape
    scale = lr * math.sqrt(max(1.0, rows / cols))
    tol = scale * 4.3 ** steps * 8 * 2.0 ** -22 * (1 + math.sqrt(min(rows, cols)) / 8) + 2 * U * float(want.norm())
    err = float((t[0].double() - want).norm())
    assert err <= tol, (err, tol, err / scale / float(x.norm()))
    assert ((t[3].double() - m).abs() <= 2 * U * (m.abs() + before[2].abs().double())).all()
    assert torch.equal(t[2], before[2])
    if t[1] is not None:
        assert torch.equal(t[1], t[0].to(torch.bfloat16))
    return err / scale / max(float(x.norm()), 1e-30)


def copies(t):
    return tuple(None if v is None else v.clone() for v in t)


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (8, 64), (64, 27), (64, 64), (65, 63), (128, 576), (127, 1000), (129, 129), (256, 256), (257, 300),
          (300, 257), (256, 2304), (513, 1000), (1000, 513), (33, 4097), (2000, 5), (640, 700)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_update(p, rows, cols):
    for nesterov, decay in ((True, 0.01), (False, 0.0)):
        t = tensors(rows, cols, seed=rows + cols)
        before = copies(t)
        run(p, [t], decay=decay, nesterov=nesterov)
        check(t, before, 0.02, 0.95, decay, 5, nesterov)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7, 10])
@pytest.mark.parametrize("rows,cols", [(70, 200), (200, 330), (530, 300)])
def test_steps(p, rows, cols, steps):
    t = tensors(rows, cols, seed=steps)
    before = copies(t)
    run(p, [t], steps=steps)
    check(t, before, 0.02, 0.95, 0.01, steps, True)


@pytest.mark.parametrize("rows,cols,rank", [(256, 256, None), (256, 256, 40), (200, 1500, None), (200, 1500, 30), (512, 4608, 100), (900, 300, 50)])
def test_as_close_as_fp32(p, rows, cols, rank):
    """w = 0 and lr = 1: the result is X itself, up to the factor for tall matrices."""
    torch.backends.cuda.matmul.allow_tf32 = False
    t = tensors(rows, cols, seed=7, rank=rank, w16=False)
    t[0].zero_()
    before = copies(t)
    run(p, [t], lr=1.0, decay=0.0)
    want, _, x = reference(before, 1.0, 0.95, 0.0, 5, True)
    plain, _, _ = reference(before, 1.0, 0.95, 0.0, 5, True, torch.float32)
    err = float((t[0].double() - want).norm() / want.norm())
    err32 = float((plain.double() - want).norm() / want.norm())
    print(f"{rows} x {cols} rank {rank}: {err:.2e}, plain fp32 {err32:.2e}")
    assert err <= 4 * err32 + 2.0 ** -20


def test_many_tensors_at_once(p):
    """More than one launch holds, of mixed shapes, some not 16-byte aligned, some without a bf16 copy."""
    shapes = [(3 + 7 * i % 90, 5 + 31 * i % 400) for i in range(19)] + [(300, 310), (5, 600), (600, 5), (256, 300)]
    ts = [tensors(r, c, seed=i, offset=i % 3, w16=i % 4 != 0) for i, (r, c) in enumerate(shapes)]
    before = [copies(t) for t in ts]
    run(p, ts)
    for t, b in zip(ts, before):
        check(t, b, 0.02, 0.95, 0.01, 5, True)
    # alone they come out the same, bit for bit
    for k in (0, 5, 20, 22):
        alone = copies(before[k])
        run(p, [alone], fill=0)
        assert torch.equal(alone[0], ts[k][0])


def test_repeats_bit_for_bit(p):
    t = tensors(300, 700, seed=3)
    other = copies(t)
    run(p, [t])
    run(p, [other], fill=0x11)
    assert torch.equal(t[0], other[0]) and torch.equal(t[3], other[3])


def test_what_surrounds_the_tensors_stays(p):
    for rows, cols, offset in ((7, 13, 3), (130, 264, 4), (264, 130, 1)):
        t = tensors(rows, cols, offset=offset)
        run(p, [t])
        for v in t:
            base = torch.empty(0, dtype=v.dtype, device=DEV).set_(v.untyped_storage())
            assert (base[:offset] == 77).all() and (base[offset + rows * cols:] == 77).all()


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e20])
def test_any_scale_of_gradient(p, scale):
    t = tensors(40, 90, seed=2)
    t[3].zero_()
    t[2].mul_(scale)
    before = copies(t)
    run(p, [t])
    check(t, before, 0.02, 0.95, 0.01, 5, True)


def test_zero_and_nan(p):
    zero, nan, inf, fine = (tensors(50, 60, seed=i) for i in range(4))
    zero[2].zero_(), zero[3].zero_()
    nan[2][3, 4] = math.nan
    inf[2][0, 0] = math.inf
    before = [copies(t) for t in (zero, nan, inf, fine)]
    run(p, [zero, nan, inf, fine])
    assert torch.equal(zero[0], torch.tensor(1 - float(np.float32(0.02)) * float(np.float32(0.01))).float().to(DEV) * before[0][0])
    assert torch.isnan(nan[0]).all() and torch.isnan(inf[0]).all()
    check(fine, before[3], 0.02, 0.95, 0.01, 5, True)


def test_singular_values_move_to_one(p):
    t = tensors(128, 512, seed=9, w16=False)
    t[0].zero_()
    run(p, [t], lr=1.0, decay=0.0)
    s = torch.linalg.svdvals(t[0].double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25  # the quintic's interval around one


def test_a_recorded_graph_on_another_stream(p):
    ts = [tensors(100, 260, seed=1), tensors(90, 31, seed=2)]
    table = p.vgg19_muon_tensors(ts)
    ws = torch.empty(p.vgg19_muon_workspace_bytes(table), dtype=torch.uint8, device=DEV)
    keep = [copies(t) for t in ts]
    p.vgg19_muon_update(table, 0.02, 0.95, 0.01, 5, True, ws, torch.cuda.current_stream())  # (first use outside the capture)
    for t, k in zip(ts, keep):
        for a, b in zip(t, k):
            a.copy_(b)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        p.vgg19_muon_update(table, 0.02, 0.95, 0.01, 5, True, ws, st)
    for seed in (5, 6):
        for i, t in enumerate(ts):
            t[2].copy_(gradient(*t[2].shape, seed + 10 * i))
        before = [copies(t) for t in ts]
        graph.replay()
        torch.cuda.synchronize()
        for t, b in zip(ts, before):
            check(t, b, 0.02, 0.95, 0.01, 5, True)


def test_refusals(p):
    w, w16, g, m = tensors(20, 30)
    st = torch.cuda.current_stream()

    def refused(code, fn):
        with pytest.raises(p.Vgg19Error) as e:
            fn()
        assert e.value.code == code

    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_tensors([(w.half(), None, g, m)]))
    refused(p.VGG19_ERR_SHAPE, lambda: p.vgg19_muon_tensors([(w, None, g[:10], m)]))
    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_tensors([(w, None, g.t().contiguous().t(), m)]))
    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_tensors([(w, w, g, m)]))
    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_tensors([(w, None, g.cpu(), m)]))
    t = p.vgg19_muon_tensors([(w, w16, g, m)])
    n = p.vgg19_muon_workspace_bytes(t)
    ws = torch.empty(n + 256, dtype=torch.uint8, device=DEV)
    refused(p.VGG19_ERR_WORKSPACE, lambda: p.vgg19_muon_update(t, 0.1, 0.9, 0, 5, True, ws[:n - 1], st))
    refused(p.VGG19_ERR_WORKSPACE, lambda: p.vgg19_muon_update(t, 0.1, 0.9, 0, 5, True, ws[1:], st))
    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_update(t, 0.1, 0.9, 0, 0, True, ws, st))
    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_update(t, math.nan, 0.9, 0, 5, True, ws, st))
    refused(p.VGG19_ERR_ARG, lambda: p.vgg19_muon_update(t, 0.1, 0.9, 0, 5, True, ws.cpu(), st))
    p.vgg19_muon_update([], 0.1, 0.9, 0, 5, True, ws, st)


@pytest.mark.parametrize("dtype_name", ["bf16", "fp32"])
def test_network_step(p, dtype_name):
    """Every parameter of a network, and that the passes after it run on the new ones."""
    import seeded_inputs as si
    dtype = p.VGG19_BF16 if dtype_name == "bf16" else p.VGG19_FP32
    params = si.vgg19_params(32, 32, seed=0, bias_std=0.1, bf16_exact=True)
    net = p.Net(32, 32, 2, dtype, params=params)
    images = torch.from_numpy(si.images(2, 32, 32, seed=1, bf16_exact=True)).to(DEV).to(net.act_dtype)
    labels = torch.from_numpy(si.labels(2, seed=2)).to(DEV)
    grads, _ = net.backward(images, labels)
    grads = grads.clone()
    momentum = torch.zeros_like(grads)
    net.muon_step(grads, momentum, 0.02, decay=0.01, bias_lr=0.1)
    p.vgg19_ops_status(torch.cuda.current_stream())
    got = np.empty(net.n_params, dtype=np.float32)
    p.vgg19_get_params(net.handle, got)
    old, new = torch.from_numpy(params).to(DEV), torch.from_numpy(got).to(DEV)
    for off, dims in net.param_slices():
        n = int(np.prod(dims))
        part = [v[off:off + n] for v in (old, new, grads, momentum)]
        if len(dims) == 1:
            want = part[0].double() - 0.1 * (1 + 0.95) * part[2].double()
            assert ((part[1].double() - want).abs() <= 4 * U * (part[0].double().abs() + 0.2 * part[2].double().abs())).all()
            assert torch.equal(part[3], part[2])
        else:
            shape = (dims[0], n // dims[0])
            o, w, g, m = (v.view(shape) for v in part)
            check((w, None, g, m), (o, None, g, torch.zeros_like(m)), 0.02, 0.95, 0.01, 5, True)
    again = p.Net(32, 32, 2, dtype, params=got)
    a, _ = net.backward(images, labels)
    b, _ = again.backward(images, labels)
    assert torch.equal(a, b)
    assert torch.equal(net.forward(images), again.forward(images))
    with pytest.raises(p.Vgg19Error):
        net.muon_step(grads, momentum[:-1], 0.02)
    net.close(), again.close()


def test_elements_beyond_32_bits(p):
    """130 x 2^24: the last row's end is beyond 2^31 elements.  Columns without gradient take no part, so the first and the last
    thousand are those of the matrix that has only them, and what lies between decays."""
    rows, cols, k = 130, 1 << 24, 1000
    small = tensors(rows, 2 * k, seed=4)
    before = copies(small)
    wide = (torch.ones(rows, cols, device=DEV), torch.ones(rows, cols, device=DEV, dtype=torch.bfloat16), torch.zeros(rows, cols, device=DEV),
            torch.zeros(rows, cols, device=DEV))
    for a, b in zip(wide, small):
        a[:, :k], a[:, -k:] = b[:, :k], b[:, k:]
    run(p, [wide], lr=0.02, decay=0.01)
    got = tuple(torch.cat([a[:, :k], a[:, -k:]], 1) for a in wide)
    check(got, before, 0.02, 0.95, 0.01, 5, True)
    decayed = torch.tensor(1 - 0.02 * 0.01, device=DEV)
    for c0 in range(k, cols - k, 1 << 20):
        between = wide[0][:, c0:min(c0 + (1 << 20), cols - k)]
        assert (between - decayed).abs().max() <= 2 * U
    assert not wide[3][:, k:-k].any()


def test_one_gradient_for_two_matrices(p):
    t = tensors(90, 200, seed=6)
    other = copies(t)[:2] + (t[2], copies(t)[3])
    before = copies(t)
    run(p, [t, other])
    check(t, before, 0.02, 0.95, 0.01, 5, True)
    assert torch.equal(t[0], other[0]) and torch.equal(t[3], other[3])
    for bad in ([t, t], [t, other[:3] + (t[3],)], [(t[0], None, t[0], t[3])]):
        with pytest.raises(p.Vgg19Error) as e:
            run(p, bad)
        assert e.value.code == p.VGG19_ERR_ARG


def test_two_recorded_graphs_share_a_workspace(p):
    """Replayed in turn on one stream, as the documentation asks."""
    ts = [tensors(150, 400, seed=8), tensors(300, 64, seed=9)]
    want = [copies(t) for t in ts]
    tables = [p.vgg19_muon_tensors([t]) for t in ts]
    ws = torch.empty(max(p.vgg19_muon_workspace_bytes(t) for t in tables), dtype=torch.uint8, device=DEV)
    st = torch.cuda.Stream()
    graphs = []
    for table in tables:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            p.vgg19_muon_update(table, 0.02, 0.95, 0.01, 5, True, ws, stream=st)
        graphs.append(graph)
    for _ in range(3):
        for graph, w in zip(graphs, want):
            graph.replay()
            run(p, [w])
    torch.cuda.synchronize()
    for t, w in zip(ts, want):
        assert torch.equal(t[0], w[0]) and torch.equal(t[3], w[3])


@pytest.mark.parametrize("rows,cols", [(1025, 1025), (1100, 1300), (1290, 3000), (2048, 2048), (1700, 1410)])
def test_symmetric_products_of_many_tiles(p, rows, cols):
    t = tensors(rows, cols, seed=rows)
    before = copies(t)
    run(p, [t])
    check(t, before, 0.02, 0.95, 0.01, 5, True)


def test_many_tiles_alone_and_together(p):
    """Alone the tiles are halves, together whole ones: the same, bit for bit."""
    ts = [tensors(1100 + 90 * i, 1500, seed=i) for i in range(5)]
    before = [copies(t) for t in ts]
    run(p, ts)
    for k in (0, 3):
        alone = copies(before[k])
        run(p, [alone], fill=0)
        assert torch.equal(alone[0], ts[k][0])


def test_network_step_refuses_a_workspace_over_the_last_bias(p):
    """The update's tensors are the weights; a workspace that begins in the last bias's momentum meets none of them."""
    net = p.Net(32, 32, 1, p.VGG19_BF16, seed=1)
    n, need = net.n_params * 4, p.vgg19_muon_step_bytes(net.handle)
    memory = torch.zeros(n + need, dtype=torch.uint8, device=DEV)
    momentum, grads = memory[:n].view(torch.float32), torch.zeros(net.n_params, device=DEV)
    ws = memory[(n - 3000) // 256 * 256:]
    assert ws.data_ptr() >= momentum.data_ptr() + 4 * net.param_slices()[37][0] and ws.numel() >= need
    for g, m, w in ((grads, momentum, ws), (momentum, momentum, torch.empty(need, dtype=torch.uint8, device=DEV)),
                    (ws[:n].view(torch.float32), momentum, torch.empty(need, dtype=torch.uint8, device=DEV))):
        with pytest.raises(p.Vgg19Error) as e:
            p.vgg19_muon_step(net.handle, g, m, 0.1, 0.9, 0.0, 0.1, 5, True, w, w.numel(), torch.cuda.current_stream())
        assert e.value.code == p.VGG19_ERR_ARG and "overlap" in str(e.value)
    net.close()


def typical_bound(u, steps):
    """What errors of 8 * 2^-22 of X a step become, relative to the last X.  In the singular vectors of X: the error of a singular value, taken as one
    sign all along, since the tensor core truncates its sums, grows by f'(s); one between singular values i and j by the divided difference
    of f or (its antisymmetric part) of f(s_i) + f(s_j) over s_i + s_j, taken as independent from step to step."""
    x = u.double() / u.double().norm()
    x = x if x.shape[0] <= x.shape[1] else x.T
    orbit = [torch.linalg.eigvalsh(x @ x.T).clamp_min(0).sqrt()]
    for _ in range(steps):
        s = orbit[-1]
        orbit.append(A * s + B * s ** 3 + C * s ** 5)
    eta, own, grow, pairs, between = 8 * 2.0 ** -22, 0.0, 1.0, 1.0, 0.0
    for s, y in zip(reversed(orbit[:-1]), reversed(orbit[1:])):
        own = own + eta * y.abs() * grow
        between += (eta * float(y.norm())) ** 2 * (float((pairs ** 2).mean()) if torch.is_tensor(pairs) else 1.0)
        slope = (A + 3 * B * s ** 2 + 5 * C * s ** 4).abs()
        grow = grow * slope
        d = s[:, None] - s[None]
        near = d.abs() < 1e-9
        divided = torch.where(near, slope[:, None], ((y[:, None] - y[None]) / torch.where(near, 1.0, d)).abs())
        pairs = pairs * torch.maximum(divided, ((y[:, None] + y[None]) / (s[:, None] + s[None])).abs())
    return math.sqrt(float(own.square().sum()) + between) / float(orbit[-1].norm())


@pytest.mark.parametrize("steps", [5, 6, 8, 10, 13, 16])
@pytest.mark.parametrize("rows,cols,rank", [(70, 200, None), (200, 330, None), (530, 300, None), (200, 330, 30), (530, 300, 30), (1290, 3000, None), (3000, 1290, None),
                                            (2048, 2048, None), (1290, 3000, 100), (2048, 2048, 100)])
def test_the_direction_itself(p, rows, cols, rank, steps):
    """w = 0 and lr = 1: the result is X.  Gaussian gradients within the bound above; those of low rank with noise, whose small singular values amplify
    what is lost on the large ones, within four times plain fp32, the ratio of the operands' steps."""
    torch.backends.cuda.matmul.allow_tf32 = False
    t = tensors(rows, cols, seed=7, rank=rank, w16=False)
    t[0].zero_()
    before = copies(t)
    run(p, [t], lr=1.0, decay=0.0, steps=steps)
    want, m, _ = reference(before, 1.0, 0.95, 0.0, steps, True)
    err = float((t[0].double() - want).norm() / want.norm())
    if rank is None:
        tol = typical_bound(before[2].double() + 0.95 * m, steps)
    else:
        plain, _, _ = reference(before, 1.0, 0.95, 0.0, steps, True, torch.float32)
        tol = 4 * float((plain.double() - want).norm() / want.norm()) + 2.0 ** -20
    print(f"{rows} x {cols} rank {rank}, {steps} steps: {err:.2e}, bound {tol:.2e}")
    assert tol < 0.01
    assert err <= tol


@pytest.mark.parametrize("rows,cols,rank", [(1290, 3000, None), (2048, 2048, None), (2048, 2048, 100), (3000, 1290, 100), (4096, 4096, None), (4096, 4096, 100)])
def test_as_close_as_fp32_at_the_size_of_dense_layers(p, rows, cols, rank):
    """Chains of four stages, tiles on and above the diagonal: held to what test_as_close_as_fp32 asks of smaller matrices."""
    test_as_close_as_fp32(p, rows, cols, rank)
