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


@pytest.mark.parametrize("over,code", [
    (dict(x=None), "ARG"), (dict(dtype=5), "ARG"), (dict(rows=-1), "SHAPE"), (dict(rows=(1 << 20) + 1), "SHAPE"), (dict(in_=0), "SHAPE"),
    (dict(in_=(1 << 24) + 1), "SHAPE"), (dict(out=0), "SHAPE"), (dict(ldx=99), "SHAPE"), (dict(group=16), "ARG"), (dict(codes=None), "ARG"),
    (dict(scales=None), "ARG"), (dict(codes=SOME + 8), "ARG"), (dict(scales=SOME + 2), "ARG"), (dict(y=None, y_f32=None), "ARG"),
    (dict(x=SOME + 1), "ARG"), (dict(bias=SOME + 2), "ARG"), (dict(y_f32=SOME + 2), "ARG")])
def test_q4_linear_refuses(p, over, code):
    a = dict(x=SOME, dtype=1, rows=2, in_=100, ldx=100, codes=SOME, scales=SOME, out=10, group=32, bias=SOME, relu=0, y=SOME,
             y_f32=SOME, stream=None)
    a.update(over)
    assert p.binding.load().vgg19_q4_linear(*a.values()) == getattr(p, "VGG19_ERR_" + code)


@pytest.mark.parametrize("over,code", [
    (dict(w=None), "ARG"), (dict(dtype=-1), "ARG"), (dict(out=0), "SHAPE"), (dict(in_=0), "SHAPE"), (dict(ld=99), "SHAPE"),
    (dict(group=100), "ARG"), (dict(codes=None), "ARG"), (dict(scales=None), "ARG"), (dict(w=SOME + 1), "ARG"),
    (dict(out=1 << 24, in_=1 << 24, ld=1 << 24), "SHAPE")])
def test_q4_pack_refuses(p, over, code):
    a = dict(w=SOME, dtype=0, out=10, in_=100, ld=100, group=32, codes=SOME, scales=SOME, stream=None)
    a.update(over)
    assert p.binding.load().vgg19_q4_pack(*a.values()) == getattr(p, "VGG19_ERR_" + code)


def test_q4_sizes(p):
    assert p.vgg19_q4_code_bytes(1, 1) == 1024 and p.vgg19_q4_code_bytes(17, 129) == 4 * 1024
    assert p.vgg19_q4_scale_bytes(1, 1, 128) == 32 and p.vgg19_q4_scale_bytes(17, 129, 32) == 4 * 128
    assert p.vgg19_q4_code_bytes(0, 5) == 0 and p.vgg19_q4_scale_bytes(5, 5, 48) == 0


def test_q4_configuration(p):
    import ctypes
    out = ctypes.c_void_p()
    cfg = p.binding.vgg19_config(32, 32, 1, p.VGG19_FP32, p.VGG19_FLAG_SPLIT_F16 | p.VGG19_FLAG_DENSE_Q4)
    assert p.binding.load().vgg19_create(ctypes.byref(cfg), 0, ctypes.byref(out)) == p.VGG19_ERR_ARG


@pytest.mark.parametrize("over,code", [
    (dict(count=-1), "ARG"), (dict(rows=0), "SHAPE"), (dict(cols=1 << 25), "SHAPE"), (dict(rows=40000, cols=40000), "SHAPE"), (dict(w=None), "ARG"),
    (dict(grad=None), "ARG"), (dict(momentum_=None), "ARG"), (dict(w=SOME + 2), "ARG"), (dict(w16=SOME + 1), "ARG"), (dict(steps=0), "ARG"),
    (dict(steps=17), "ARG"), (dict(lr=float("nan")), "ARG"), (dict(decay=float("nan")), "ARG"), (dict(ws=None), "WORKSPACE"),
    (dict(ws=SOME + 16), "WORKSPACE"), (dict(nbytes=100), "WORKSPACE")])
def test_muon_update_refuses(p, over, code):
    a = dict(w=SOME, w16=SOME, grad=SOME, momentum_=SOME, rows=30, cols=50, count=1, lr=0.1, mu=0.9, decay=0.0, steps=5, ws=SOME, nbytes=1 << 40)
    a.update(over)
    t = (p.binding.vgg19_muon_tensor * 1)()
    t[0].w, t[0].w_bf16, t[0].grad, t[0].momentum, t[0].rows, t[0].cols = a["w"], a["w16"], a["grad"], a["momentum_"], a["rows"], a["cols"]
    rc = p.binding.load().vgg19_muon_update(t, a["count"], a["lr"], a["mu"], a["decay"], a["steps"], 1, a["ws"], a["nbytes"], None)
    assert rc == getattr(p, "VGG19_ERR_" + code)


def test_muon_sizes(p):
    t = (p.binding.vgg19_muon_tensor * 1)()
    t[0].rows, t[0].cols = 100, 1000
    lib = p.binding.load()
    one = lib.vgg19_muon_workspace_bytes(t, 1)
    assert one >= 2 * 2 * 2 * 100 * 1000 + 5 * 2 * 2 * 100 * 104
    t[0].rows, t[0].cols = 1000, 100
    assert lib.vgg19_muon_workspace_bytes(t, 1) == one
    t[0].rows = 0
    assert lib.vgg19_muon_workspace_bytes(t, 1) == 0
    assert lib.vgg19_muon_update(None, 0, 0.1, 0.9, 0.0, 5, 1, None, 0, None) == p.VGG19_OK
    assert lib.vgg19_muon_step(None, None, None, 0.1, 0.9, 0.0, 0.1, 5, 1, None, 0, None) == p.VGG19_ERR_ARG
    assert lib.vgg19_muon_step_bytes(None) == 0


@pytest.mark.parametrize("where", ["ids", "logprob", "lse", "entropy", "top_id", "top_logprob"])
def test_logprobs_refuses_unaligned_words(p, where):
    assert p.binding.load().vgg19_logprobs(*logprobs_args(**{where: SOME + 2})) == p.VGG19_ERR_ARG


def backward_args(**over):
    a = dict(logits=SOME, dtype=0, rows=3, classes=10, ld=24, ids=SOME, n_ids=1, lse=SOME, entropy=SOME, d_logprob=SOME,
             d_entropy=SOME, d_logits=SOME, d_ld=24, stream=None)
    a.update(over)
    return a.values()


@pytest.mark.parametrize("where", ["ids", "lse", "entropy", "d_logprob", "d_entropy"])
def test_logprobs_backward_refuses_unaligned_words(p, where):
    assert p.binding.load().vgg19_logprobs_backward(*backward_args(**{where: SOME + 2})) == p.VGG19_ERR_ARG


# Gradients over other logits than their own: shifted within the row, rows of another stride, one row further.
@pytest.mark.parametrize("over", [
    dict(d_logits=SOME + 4), dict(d_logits=SOME - 4), dict(d_ld=25), dict(d_ld=10), dict(d_logits=SOME + 4 * 24), dict(d_logits=SOME + 4 * 9),
    dict(d_logits=SOME + 4 * 15), dict(rows=1, d_logits=SOME + 4 * 9), dict(d_logits=SOME + 4 * 57, d_ld=30)])
def test_logprobs_backward_refuses_overlaps(p, over):
    assert p.binding.load().vgg19_logprobs_backward(*backward_args(**over)) == p.VGG19_ERR_ARG
    assert "overlap" in p.vgg19_last_error()


@pytest.mark.parametrize("over", [
    dict(y=SOME), dict(y=SOME + 2 * 99), dict(y=SOME - 2 * 19), dict(y_f32=SOME + 2 * 200), dict(y=SOME + 2 * 101), dict(y=SOME + 4 * 1000, y_f32=SOME + 4 * 1000),
    dict(rows=1, y=SOME + 2 * 99)])
def test_q4_linear_refuses_overlaps(p, over):
    a = dict(x=SOME, dtype=1, rows=2, in_=100, ldx=116, codes=SOME, scales=SOME, out=10, group=32, bias=SOME, relu=0, y=None,
             y_f32=None, stream=None)
    a.update(over)
    assert p.binding.load().vgg19_q4_linear(*a.values()) == p.VGG19_ERR_ARG
    assert "overlap" in p.vgg19_last_error()


# 30 x 50 matrices: 6000 bytes of fp32, 3000 of bf16; places are multiples of 8000 but for what each case changes.
@pytest.mark.parametrize("change", [
    {(0, "w"): 5}, {(0, "w_bf16"): 0.5}, {(1, "grad"): 0}, {(0, "grad"): 3}, {(1, "momentum"): 3}, {(1, "w_bf16"): 1}, {(1, "grad"): 5.9 / 8}, {(0, "w"): 9},
    {(0, "momentum"): 7.7}])
def test_muon_update_refuses_overlaps(p, change):
    t = (p.binding.vgg19_muon_tensor * 2)()
    for i in range(2):
        t[i].rows, t[i].cols = 30, 50
        for k, name in enumerate(("w", "w_bf16", "grad", "momentum")):
            setattr(t[i], name, SOME + int(8000 * change.get((i, name), 4 * i + k)))
    lib = p.binding.load()
    ws = SOME + 9 * 8000 // 256 * 256
    rc = lib.vgg19_muon_update(t, 2, 0.1, 0.9, 0.0, 5, 1, ws if (0, "w") in change else 1 << 30, 1 << 40, None)
    assert rc == p.VGG19_ERR_ARG and "overlap" in p.vgg19_last_error()


def test_the_binding_refuses_sizes_beyond_an_int(p):
    wide = torch.empty(1, (1 << 32) + 5, device="meta")
    for call in (lambda: p.vgg19_logprobs(wide), lambda: p.vgg19_q4_pack(wide, 64, None, None), lambda: p.vgg19_muon_tensors([(wide, None, wide, wide)])):
        with pytest.raises(p.Vgg19Error) as e:
            call()
        assert e.value.code == p.VGG19_ERR_SHAPE


@pytest.mark.parametrize("which,ws,nbytes,code", [(-1, SOME, 1 << 20, "ARG"), (3, SOME, 1 << 20, "ARG"), (0, None, 1 << 20, "WORKSPACE"),
                                                  (1, SOME + 16, 1 << 20, "WORKSPACE"), (2, SOME, (1 << 20) - 1, "WORKSPACE")])
def test_the_operators_selftest_refuses(p, which, ws, nbytes, code):
    assert p.binding.load().vgg19_selftest_operator_timeout(None, which, ws, nbytes, None) == getattr(p, "VGG19_ERR_" + code)
    assert p.VGG19_SELFTEST_BYTES == 1 << 20


# 3 rows of 10 fp32 logits, 24 apart; 2 ids and the best 4 of each row; every array on its own 4096 bytes but for what a case changes.
def apart(**over):
    names = ("logits", "ids", "logprob", "lse", "entropy", "top_id", "top_logprob")
    a = dict(dtype=0, rows=3, classes=10, ld=24, n_ids=2, top_k=4, **{n: SOME + 4096 * i for i, n in enumerate(names)})
    a.update({k: SOME + v for k, v in over.items()})
    return logprobs_args(**a)


@pytest.mark.parametrize("over", [
    dict(lse=0), dict(logprob=4 * 9), dict(entropy=4 * 8), dict(top_id=-4 * 11), dict(top_logprob=4 * 57), dict(lse=4 * 24 + 4 * 22), dict(lse=4096 + 20),
    dict(logprob=4096 - 20), dict(entropy=3 * 4096 + 8), dict(top_id=6 * 4096 + 44), dict(lse=2 * 4096 + 20), dict(top_logprob=4 * 4096 - 44)])
def test_logprobs_refuses_overlaps(p, over):
    assert p.binding.load().vgg19_logprobs(*apart(**over)) == p.VGG19_ERR_ARG
    assert "overlap" in p.vgg19_last_error()


# rows of 24 with ids, sums or gradients of the results between or in them
@pytest.mark.parametrize("over", [
    dict(lse=SOME + 40960), dict(entropy=SOME + 40960 + 4 * 33), dict(d_logprob=SOME + 40960 + 4 * 57), dict(ids=SOME + 40960 - 4), dict(d_entropy=SOME + 40960 + 4 * 8)])
def test_logprobs_backward_refuses_inputs_in_its_gradient(p, over):
    a = dict(ids=SOME + 4096, lse=SOME + 8192, entropy=SOME + 12288, d_logprob=SOME + 16384, d_entropy=SOME + 20480, d_logits=SOME + 40960)
    a.update(over)
    assert p.binding.load().vgg19_logprobs_backward(*backward_args(**a)) == p.VGG19_ERR_ARG
    assert "overlap" in p.vgg19_last_error()


# 10 x 100 weights in groups of 32: 1024 bytes of codes, 128 of scales; two rows of x
@pytest.mark.parametrize("over", [dict(y=8192 + 1020), dict(y=8192 - 36), dict(y_f32=12288 + 124), dict(y_f32=12288 - 76), dict(y=16384 + 36), dict(y_f32=16384 - 76)])
def test_q4_linear_refuses_outputs_over_weights(p, over):
    a = dict(x=0, dtype=1, rows=2, in_=100, ldx=116, codes=8192, scales=12288, out=10, group=32, bias=16384, relu=0, y=20480, y_f32=24576, stream=None)
    a.update(over)
    for k in ("x", "codes", "scales", "bias", "y", "y_f32"):
        a[k] += SOME
    assert p.binding.load().vgg19_q4_linear(*a.values()) == p.VGG19_ERR_ARG
    assert "overlap" in p.vgg19_last_error()


@pytest.mark.parametrize("over", [dict(codes=0), dict(codes=3968), dict(codes=5120 - 1008), dict(scales=8192 + 1008), dict(scales=8192 - 112), dict(scales=1056), dict(scales=4096 + 3888)])
def test_q4_pack_refuses_overlaps(p, over):
    a = dict(w=4096, dtype=0, out=10, in_=100, ld=100, group=32, codes=8192, scales=12288, stream=None)
    a.update({k: v + (4096 if v < 4096 else 0) for k, v in over.items()})
    for k in ("w", "codes", "scales"):
        a[k] += SOME
    assert p.binding.load().vgg19_q4_pack(*a.values()) == p.VGG19_ERR_ARG
    assert "overlap" in p.vgg19_last_error()


def test_the_operators_selftest_refuses_host_memory(p):
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_selftest_operator_timeout(None, p.VGG19_SELFTEST_UPDATE, torch.empty(1 << 20, dtype=torch.uint8))
    assert e.value.code == p.VGG19_ERR_ARG
