"""Dense layers over 4-bit weights against plain arithmetic in 64 bits on the same codes.

Tolerances.  With u = 2^-24: a product of a code and a bf16 term is exact; fp32 activations are exact sums of three terms (below
2^-126 they may be lost).  The sums run in fp32 in some order that the tensor core is free in, truncating: at most 2 u per
addition, of partial sums no larger than A = sum |x| |code - 8| scale.  Additions on the longest chain: the terms of a group (at
most 3 x 8 instructions of 16), the groups of a warp's share (in / 128 blocks over at least one warp), eight to join.  So
2 u (24 + 16 + in / 32 + 16) A, the rounding of the bias sum, and half a step of the result's type."""
import math

import numpy as np
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


def buffers(p, out, in_, group, fill=0x5a):
    codes = torch.full((p.vgg19_q4_code_bytes(out, in_),), fill, dtype=torch.uint8, device=DEV)
    scales = torch.full((p.vgg19_q4_scale_bytes(out, in_, group) // 2,), float("nan"), dtype=torch.bfloat16, device=DEV)
    return codes, scales


def decode(codes, scales, out, in_, group):
    """(integers [out][in], scales [out][in]) of the documented layout, one weight at a time."""
    tiles, blocks = -(-out // 16), -(-in_ // 128)
    c = codes.cpu().numpy().reshape(tiles, blocks, 16, 16, 4)
    s = scales.float().cpu().numpy().reshape(tiles, blocks, 16, 128 // group)
    k = np.arange(in_)
    o = np.arange(out)[:, None]
    kk = k % 128
    u, t, j = kk // 32, kk % 32 // 8, kk % 8
    byte = c[o // 16, k // 128, o % 16, 4 * t + u, j // 2]
    q = (byte >> (4 * (j % 2))) & 15
    return q.astype(np.int64) - 8, s[o // 16, k // 128, o % 16, kk // group].astype(np.float64)


def expected_pack(w, group):
    """By the definition, group by group, in fp32 where the definition rounds."""
    w = w.float().cpu()
    out, in_ = w.shape
    q = torch.zeros(out, in_)
    s = torch.zeros(out, in_)
    for a in range(0, in_, group):
        part = w[:, a:a + group].numpy()
        amax = np.abs(part).max(1, keepdims=True)
        sc = torch.from_numpy((amax / np.float32(7)).astype(np.float32)).to(torch.bfloat16).float().numpy()
        with np.errstate(divide="ignore", invalid="ignore"):
            r = np.where(sc > 0, np.rint(part / sc), 0)
        q[:, a:a + group] = torch.from_numpy(np.clip(r, -8, 7))
        s[:, a:a + group] = torch.from_numpy(np.broadcast_to(sc, part.shape).copy())
    return q.numpy().astype(np.int64), s.numpy().astype(np.float64)


def weights(out, in_, dtype="fp32", seed=0, ld=None, offset=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ld = ld or in_
    buf = torch.full((offset + out * ld,), float("nan"), dtype=TYPES[dtype], device=DEV)
    w = buf[offset:].view(out, ld)[:, :in_]
    w.copy_(torch.randn(out, in_, generator=gen, device=DEV) * math.sqrt(2.0 / in_))
    return w


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("out,in_,group,ld,offset", [(1, 1, 32, 1, 0), (16, 128, 128, 128, 0), (17, 129, 64, 131, 1), (40, 300, 32, 300, 3),
                                                     (1000, 4096, 64, 4096, 0), (5, 1000, 128, 1001, 0)])
def test_pack(p, out, in_, group, ld, offset, dtype):
    w = weights(out, in_, dtype, seed=out, ld=ld, offset=offset)
    w[0] = 0
    if out > 2 and in_ > 2:
        w[1, 0], w[2, 1] = 100.0, -1e-39
    codes, scales = buffers(p, out, in_, group)
    p.vgg19_q4_pack(w, group, codes, scales, torch.cuda.current_stream())
    q, s = decode(codes, scales, out, in_, group)
    want_q, want_s = expected_pack(w, group)
    assert np.array_equal(s, want_s) and np.array_equal(q, want_q)
    # the padding: finite scales of zero and codes of eight
    tiles, blocks = -(-out // 16), -(-in_ // 128)
    full_q, full_s = decode(codes, scales, tiles * 16, blocks * 128, group)
    assert not full_q[out:].any() and not full_q[:, in_:].any() and np.isfinite(full_s).all() and not full_s[out:].any()


def inputs(rows, in_, dtype, seed=1, ld=None, offset=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ld = ld or in_
    buf = torch.full((offset + rows * ld + 16,), float("nan"), dtype=TYPES[dtype], device=DEV)
    x = buf[offset:offset + rows * ld].view(rows, ld)[:, :in_]
    x.copy_(torch.randn(rows, in_, generator=gen, device=DEV))
    return x


def reference(x, codes, scales, out, group, bias, relu):
    q, s = decode(codes, scales, out, x.shape[1], group)
    w = torch.from_numpy(q * s)
    x64 = x.double().cpu()
    y = x64 @ w.T + (0 if bias is None else bias.double().cpu())
    size = x64.abs() @ w.abs().T + (0 if bias is None else bias.double().cpu().abs())
    return (y.clamp_min(0) if relu else y), size


def within(got, want, size, in_):
    tol = 2 * U * (56 + in_ / 32) * size
    half = {torch.float32: U, torch.bfloat16: 2.0 ** -8}[got.dtype]
    return bool(((got.double().cpu() - want).abs() <= tol + half * want.abs()).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,out,in_,group,relu", [
    (1, 1, 1, 32, False), (1, 16, 128, 128, True), (2, 15, 127, 64, False), (3, 17, 129, 32, True), (8, 100, 1000, 128, False),
    (9, 33, 640, 64, True), (16, 1000, 4096, 128, False), (5, 4099, 5003, 64, False), (1, 4096, 25088, 64, True), (17, 48, 300, 32, False),
    (40, 31, 257, 64, True), (16, 64, 25088, 32, False), (13, 2048, 1025, 32, False)])
def test_linear(p, rows, out, in_, group, relu, dtype):
    w = weights(out, in_, seed=out + in_)
    codes, scales = buffers(p, out, in_, group)
    st = torch.cuda.current_stream()
    p.vgg19_q4_pack(w, group, codes, scales, st)
    x = inputs(rows, in_, dtype, seed=rows)
    bias = torch.randn(out, generator=torch.Generator(device=DEV).manual_seed(9), device=DEV) * 0.1
    y = torch.full((rows, out), float("nan"), dtype=x.dtype, device=DEV)
    yf = torch.full((rows, out), float("nan"), dtype=torch.float32, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, bias, relu, y, yf, st)
    want, size = reference(x, codes, scales, out, group, bias, relu)
    assert within(yf, want, size, in_)
    assert within(y, want, size, in_)
    assert torch.equal(y, yf.to(y.dtype))
    again = torch.empty_like(yf)
    p.vgg19_q4_linear(x, codes, scales, out, group, bias, relu, None, again, st)
    assert torch.equal(again, yf)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("ld,offset", [(500, 0), (501, 1), (512, 3), (1024, 8)])
def test_strides_and_starts(p, ld, offset, dtype):
    out, in_, group = 70, 500, 32
    codes, scales = buffers(p, out, in_, group)
    st = torch.cuda.current_stream()
    p.vgg19_q4_pack(weights(out, in_), group, codes, scales, st)
    x = inputs(6, in_, dtype, ld=ld, offset=offset)
    y = torch.empty(6, out, dtype=x.dtype, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, None, False, y, None, st)
    want, size = reference(x, codes, scales, out, group, None, False)
    assert within(y, want, size, in_)


def test_every_code_and_place(p):
    """x a unit vector per row: each weight comes out by itself, exactly."""
    out, in_, group = 32, 256, 64
    gen = torch.Generator(device=DEV).manual_seed(4)
    codes = torch.randint(0, 256, (p.vgg19_q4_code_bytes(out, in_),), generator=gen, device=DEV, dtype=torch.uint8)
    scales = (torch.rand(p.vgg19_q4_scale_bytes(out, in_, group) // 2, generator=gen, device=DEV) + 0.5).to(torch.bfloat16)
    x = torch.eye(in_, device=DEV)
    y = torch.empty(in_, out, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, y=y, stream=torch.cuda.current_stream())
    q, s = decode(codes, scales, out, in_, group)
    assert np.array_equal(y.cpu().numpy().T.astype(np.float64), q * s)
    assert set(np.unique(q)) == set(range(-8, 8))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_infinities_and_nans(p, dtype):
    out, in_, group = 33, 400, 32
    w = weights(out, in_)
    w[3, 100], w[4, 7] = math.nan, math.inf
    codes, scales = buffers(p, out, in_, group)
    st = torch.cuda.current_stream()
    p.vgg19_q4_pack(w, group, codes, scales, st)
    x = inputs(3, in_, dtype)
    clean = torch.empty(3, out, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, None, True, None, clean, st)
    nan = torch.isnan(clean).cpu()
    assert nan[:, 3].all() and nan[:, 4].all() and nan.sum() == 6
    # a NaN in one row of x makes that row NaN and leaves the others
    x[1, 399] = math.nan
    y = torch.empty(3, out, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, None, True, None, y, st)
    assert torch.isnan(y[1]).all()
    keep = [c for c in range(out) if c not in (3, 4)]
    assert torch.equal(y[0::2][:, keep], clean[0::2][:, keep])
    # an infinity times the weights that are not zero
    x[1, 399] = math.inf
    p.vgg19_q4_linear(x, codes, scales, out, group, None, False, None, y, st)
    q, _ = decode(codes, scales, out, in_, group)
    got = y[1].cpu().numpy()
    for c in keep:
        v = q[c, 399]
        assert (np.isnan(got[c]) if v == 0 else got[c] == (math.inf if v > 0 else -math.inf))


def test_the_largest_activations(p):
    """bf16 and fp32 values at the end of their range, which a rounded first term would turn into infinities."""
    out, in_, group = 16, 128, 128
    codes, scales = buffers(p, out, in_, group)
    w = torch.zeros(out, in_, device=DEV)
    w[:, 5] = 7 * 2.0 ** -20
    st = torch.cuda.current_stream()
    p.vgg19_q4_pack(w, group, codes, scales, st)
    for dt in TYPES.values():
        x = torch.zeros(1, in_, dtype=dt, device=DEV)
        x[0, 5] = torch.finfo(dt).max
        y = torch.empty(1, out, device=DEV)
        p.vgg19_q4_linear(x, codes, scales, out, group, None, False, None, y, st)
        assert torch.allclose(y.double(), (x[0, 5].double() * 7 * 2.0 ** -20).expand(1, out), rtol=4 * U, atol=0)


def test_a_recorded_graph_on_another_stream(p):
    out, in_, group = 200, 1000, 64
    codes, scales = buffers(p, out, in_, group)
    w = weights(out, in_)
    x = inputs(4, in_, "bf16")
    y = torch.empty(4, out, dtype=torch.bfloat16, device=DEV)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        p.vgg19_q4_pack(w, group, codes, scales, st)
        p.vgg19_q4_linear(x, codes, scales, out, group, None, False, y, None, st)
    for seed in (5, 6):
        w.copy_(weights(out, in_, seed=seed))
        x.copy_(inputs(4, in_, "bf16", seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        want, size = reference(x, codes, scales, out, group, None, False)
        assert within(y, want, size, in_)


def test_refusals(p):
    out, in_, group = 20, 200, 64
    codes, scales = buffers(p, out, in_, group)
    x = inputs(2, in_, "bf16")
    y = torch.empty(2, out, dtype=torch.bfloat16, device=DEV)
    st = torch.cuda.current_stream()

    def refused(code, fn, *a):
        with pytest.raises(p.Vgg19Error) as e:
            fn(*a)
        assert e.value.code == code

    lin = p.vgg19_q4_linear
    refused(p.VGG19_ERR_ARG, lin, x.half(), codes, scales, out, group, None, False, y, None, st)
    refused(p.VGG19_ERR_ARG, lin, x, codes.cpu(), scales, out, group, None, False, y, None, st)
    refused(p.VGG19_ERR_SHAPE, lin, x, codes[:-1], scales, out, group, None, False, y, None, st)
    refused(p.VGG19_ERR_SHAPE, lin, x, codes, scales[:-1], out, group, None, False, y, None, st)
    refused(p.VGG19_ERR_ARG, lin, x, codes, scales, out, 48, None, False, y, None, st)
    refused(p.VGG19_ERR_ARG, lin, x, codes, scales, out, group, None, False, y.float(), None, st)
    refused(p.VGG19_ERR_SHAPE, lin, x, codes, scales, out, group, torch.zeros(out + 1, device=DEV), False, y, None, st)
    refused(p.VGG19_ERR_ARG, lin, x, codes, scales, out, group, None, False, None, None, st)
    refused(p.VGG19_ERR_SHAPE, p.vgg19_q4_pack, torch.zeros(out, in_ + 128, device=DEV), group, codes, scales, st)
    lin(x[:0], codes, scales, out, group, None, False, y[:0], None, st)  # no rows, no work


# ---- a network whose dense layers answer with 4-bit weights ------------------------------------------------------

@pytest.mark.parametrize("dtype_name,batch", [("bf16", 1), ("bf16", 20), ("fp32", 3)])
def test_network_forward(p, dtype_name, batch):
    """The logits are those of a chain of 64-bit dense layers over the packed weights, from the last pool the pass stored;
    2e-2 for bf16 as the network's forward tests have it (each activation rounded by 2^-8), 1e-4 for fp32."""
    import seeded_inputs as si
    dtype = p.VGG19_BF16 if dtype_name == "bf16" else p.VGG19_FP32
    params = si.vgg19_params(32, 32, seed=0, bias_std=0.1, bf16_exact=True)
    net = p.Net(32, 32, batch, dtype, params=params, flags=p.VGG19_FLAG_DENSE_Q4, mode=p.VGG19_MODE_TRAIN)
    images = torch.from_numpy(si.images(batch, 32, 32, seed=1, bf16_exact=True)).to(DEV).to(net.act_dtype)
    logits = net.forward(images)
    net.sync_status()
    assert "4-bit" in p.vgg19_describe(net.handle)

    def check(logits, flat):
        h = net.saved_tensor(batch, p.VGG19_MODE_FORWARD, 20).reshape(batch, -1).double().cpu()
        for i in range(3):
            (wo, (o, k)), (bo, _) = net.param_slices()[32 + 2 * i], net.param_slices()[33 + 2 * i]
            q, s = expected_pack(torch.from_numpy(flat[wo:wo + o * k].reshape(o, k)), p.VGG19_DENSE_Q4_GROUP)
            h = h @ torch.from_numpy(q * s).T + torch.from_numpy(flat[bo:bo + o]).double()
            h = h.clamp_min(0) if i < 2 else h
        rel = float((logits.double().cpu() - h).norm() / h.norm())
        assert rel <= (2e-2 if dtype_name == "bf16" else 1e-4), rel

    check(logits.clone(), params)
    # the copies follow the parameters
    g = torch.zeros(net.n_params, device=DEV)
    off = net.param_slices()[32][0]
    g[off:] = torch.randn(net.n_params - off, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    net.sgd_step(g, 1e-2)
    moved = np.empty(net.n_params, dtype=np.float32)
    net.sync_status()
    p.vgg19_get_params(net.handle, moved)
    check(net.forward(images).clone(), moved)
    # and a training step, whose backward pass keeps the full weights
    labels = torch.from_numpy(si.labels(batch, seed=2)).to(DEV)
    net.train_step(images, labels, 1e-3, stream=torch.cuda.Stream())
    net.sync_status()
    torch.cuda.synchronize()
    p.vgg19_get_params(net.handle, moved)
    check(net.forward(images).clone(), moved)
    net.close()


def test_dense_layer_entry_point(p):
    import seeded_inputs as si
    params = si.vgg19_params(32, 32, seed=0, bias_std=0.1, bf16_exact=True)
    net = p.Net(32, 32, 2, p.VGG19_BF16, params=params, flags=p.VGG19_FLAG_DENSE_Q4)
    x = inputs(2, 4096, "bf16")
    y = torch.empty(2, 1000, device=DEV)
    p.vgg19_dense_layer_forward(net.handle, 3, x, 2, None, y, torch.cuda.current_stream())
    (wo, (o, k)), (bo, _) = net.param_slices()[36], net.param_slices()[37]
    q, s = expected_pack(torch.from_numpy(params[wo:wo + o * k].reshape(o, k)), p.VGG19_DENSE_Q4_GROUP)
    w, b = torch.from_numpy(q * s), torch.from_numpy(params[bo:bo + o]).double()
    want, size = x.double().cpu() @ w.T + b, x.double().cpu().abs() @ w.abs().T + b.abs()
    assert within(y, want, size, k)
    net.close()


def test_codes_beyond_32_bits(p):
    """The last rows' codes start more than 2^32 bytes after the first."""
    out, in_, group, rows = 65600, 1 << 17, 128, 2
    gen = torch.Generator(device=DEV).manual_seed(1)
    codes = torch.randint(0, 256, (p.vgg19_q4_code_bytes(out, in_),), generator=gen, dtype=torch.uint8, device=DEV)
    assert codes.numel() > 1 << 32
    scales = (torch.rand(p.vgg19_q4_scale_bytes(out, in_, group) // 2, generator=gen, device=DEV) * 0.01).to(torch.bfloat16)
    x = inputs(rows, in_, "bf16", seed=2)
    y = torch.full((rows, out), float("nan"), dtype=torch.float32, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, None, False, None, y, torch.cuda.current_stream())
    for first in (0, out // 2 // 16 * 16, out - 32):
        c = codes.view(out // 16, -1)[first // 16:first // 16 + 2].reshape(-1)
        s = scales.view(out // 16, -1)[first // 16:first // 16 + 2].reshape(-1)
        want, size = reference(x, c, s, 32, group, None, False)
        assert within(y[:, first:first + 32], want, size, in_)
    assert not torch.isnan(y).any()


# Sizes at which x takes much of a block's shared memory, and few rows of weights over a long K.
@pytest.mark.parametrize("rows,out,in_,group,dtype", [(10, 2700, 6344, 64, "fp32"), (16, 2500, 3001, 32, "bf16"), (12, 7067, 1299, 128, "bf16"), (16, 4700, 2050, 128, "fp32"),
                                                      (15, 117, 9279, 32, "fp32"), (2, 3097, 4050, 64, "bf16"), (7, 1500, 4100, 32, "fp32")])
def test_larger_sizes_for_several_rows(p, rows, out, in_, group, dtype):
    codes, scales = buffers(p, out, in_, group)
    st = torch.cuda.current_stream()
    p.vgg19_q4_pack(weights(out, in_, seed=3), group, codes, scales, st)
    x = inputs(rows, in_, dtype, seed=rows, ld=in_ + in_ % 3)
    yf = torch.full((rows, out), float("nan"), dtype=torch.float32, device=DEV)
    p.vgg19_q4_linear(x, codes, scales, out, group, None, False, None, yf, st)
    want, size = reference(x, codes, scales, out, group, None, False)
    assert within(yf, want, size, in_)
    again = torch.empty_like(yf)
    p.vgg19_q4_linear(x, codes, scales, out, group, None, False, None, again, st)
    assert torch.equal(again, yf)


@pytest.mark.parametrize("flags_name", ["recorded", "VGG19_FLAG_NO_GRAPH"])
def test_training_packs_once(p, flags_name):
    """k steps as one program pack the three dense layers once, behind the last: nothing in between reads the 4-bit copies."""
    import seeded_inputs as si
    params = si.vgg19_params(32, 32, seed=0, bf16_exact=True)
    batch, steps = 2, 3
    images = torch.from_numpy(si.images(batch * steps, 32, 32, seed=1, bf16_exact=True)).to(DEV).to(torch.bfloat16)
    labels = torch.from_numpy(si.labels(batch * steps, seed=2)).to(DEV)
    flags = 0 if flags_name == "recorded" else p.VGG19_FLAG_NO_GRAPH
    nets = [p.Net(32, 32, batch, p.VGG19_BF16, params=params, flags=f, mode=p.VGG19_MODE_TRAIN) for f in (flags, flags | p.VGG19_FLAG_DENSE_Q4)]
    losses, st, count = torch.empty(steps, device=DEV), torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for net in nets:
        p.vgg19_train_steps(net.handle, images, labels, batch, steps, 1e-3, losses, st)
        net.sync_status(st)
        count.append(p.vgg19_launch_count(net.handle, p.VGG19_MODE_TRAIN))
    assert count[1] - count[0] == 3
    flat = [np.empty(net.n_params, dtype=np.float32) for net in nets]
    for net, f in zip(nets, flat):
        p.vgg19_get_params(net.handle, f)
    assert np.array_equal(*flat) and not np.array_equal(flat[0], params)
    fresh = p.Net(32, 32, batch, p.VGG19_BF16, params=flat[1], flags=p.VGG19_FLAG_DENSE_Q4)
    assert torch.equal(nets[1].forward(images[:batch]), fresh.forward(images[:batch]))
    for net in nets + [fresh]:
        net.close()


# Sizes whose plan counts on how many blocks of a launch an SM holds.
@pytest.mark.parametrize("rows,out,in_,group,dtype", [(1, 7140, 3196, 128, "fp32"), (13, 14582, 1268, 128, "bf16"), (2, 4036, 1781, 128, "fp32"), (11, 6439, 960, 32, "bf16"),
                                                      (3, 8427, 1290, 32, "fp32"), (10, 5928, 1717, 32, "bf16")])
def test_sizes_of_more_blocks_than_fit_at_once(p, rows, out, in_, group, dtype):
    test_larger_sizes_for_several_rows(p, rows, out, in_, group, dtype)
