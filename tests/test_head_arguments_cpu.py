"""What dropout and the last layer with its loss refuse, on the host alone: every check comes before the first launch."""
import ctypes

import pytest
import torch

import __graft_entry__ as g

SOME = 1 << 20  # stands for a device address; nothing reads it
FAR = 1 << 30


@pytest.fixture(scope="module")
def p():
    g.build()
    import paper_1810_09868_b200 as pkg
    return pkg


def code_of(p, name):
    return getattr(p, "VGG19_ERR_" + name)


@pytest.mark.parametrize("over,code", [
    (dict(dtype=2), "ARG"), (dict(rows=-1), "SHAPE"), (dict(cols=0), "SHAPE"), (dict(rows=1 << 40), "SHAPE"), (dict(ldx=9), "SHAPE"), (dict(ldy=9), "SHAPE"),
    (dict(rate=-0.1), "ARG"), (dict(rate=1.5), "ARG"), (dict(rate=float("nan")), "ARG"), (dict(first=1 << 62), "ARG"), (dict(x=None), "ARG"), (dict(y=None), "ARG"),
    (dict(x=SOME + 1), "ARG"), (dict(y=FAR + 1), "ARG"), (dict(dtype=0, x=SOME + 2), "ARG"), (dict(step_counter=SOME + 4), "ARG"),
    (dict(y=SOME + 2), "ARG"), (dict(y=SOME, ldy=20), "ARG"), (dict(y=SOME - 38), "ARG"), (dict(y=SOME + 2 * 49), "ARG"), (dict(step_counter=FAR + 8), "ARG")])
def test_dropout_refuses(p, over, code):
    a = dict(x=SOME, dtype=1, rows=5, cols=10, ldx=10, rate=0.5, seed=1, step=0, step_counter=None, first=0, y=FAR, ldy=10, stream=None)
    a.update(over)
    assert p.binding.load().vgg19_dropout(*a.values()) == code_of(p, code) and p.vgg19_last_error()
    assert p.binding.load().vgg19_dropout_backward(*a.values()) == code_of(p, code)


def layer(p, **over):
    a = dict(x=SOME, ldx=64, w=SOME + (1 << 16), ldw=64, bias=SOME + (2 << 16), labels=SOME + (3 << 16), rows=5, in_=64, classes=100, dtype=1)
    a.update(over)
    return p.binding.vgg19_linear_loss(*a.values())


BAD_LAYERS = [
    (dict(dtype=2), "ARG"), (dict(rows=-1), "SHAPE"), (dict(rows=(1 << 22) + 1), "SHAPE"), (dict(in_=0), "SHAPE"), (dict(in_=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), "SHAPE"),
    (dict(rows=1 << 22, classes=1 << 23), "SHAPE"), (dict(classes=0), "SHAPE"), (dict(classes=(1 << 24) + 1), "SHAPE"), (dict(ldx=63), "SHAPE"), (dict(ldw=63), "SHAPE"), (dict(ldx=1 << 36), "SHAPE"), (dict(ldw=1 << 36), "SHAPE")]
BAD_POINTERS = [(dict(x=None), "ARG"), (dict(w=None), "ARG"), (dict(labels=None), "ARG"), (dict(x=SOME + 1), "ARG"), (dict(dtype=0, w=SOME + 2), "ARG"), (dict(labels=SOME + 2), "ARG"),
                (dict(bias=SOME + 1), "ARG")]


@pytest.mark.parametrize("over,code", BAD_LAYERS + BAD_POINTERS)
def test_layers_refused(p, over, code):
    lib, bad = p.binding.load(), layer(p, **over)
    size = lib.vgg19_linear_cross_entropy_bytes(ctypes.byref(layer(p)), 1)
    assert size > 0 and (lib.vgg19_linear_cross_entropy_bytes(ctypes.byref(bad), 0) == 0) == ((over, code) in BAD_LAYERS)
    assert lib.vgg19_linear_cross_entropy(ctypes.byref(bad), FAR, FAR + 4096, FAR + 65536, 1 << 30, None) == code_of(p, code) and p.vgg19_last_error()
    assert lib.vgg19_linear_cross_entropy_backward(ctypes.byref(bad), FAR, FAR + 4096, FAR + 8192, 64, FAR + 65536, bad.dtype, 64, None, FAR + (1 << 20), 1 << 30, None) == code_of(p, code)


def test_no_layer_is_refused(p):
    lib = p.binding.load()
    assert lib.vgg19_linear_cross_entropy_bytes(None, 0) == 0
    assert lib.vgg19_linear_cross_entropy(None, FAR, None, FAR + 256, 1 << 20, None) == p.VGG19_ERR_ARG
    assert lib.vgg19_linear_cross_entropy_backward(None, FAR, FAR, None, 0, None, 0, 0, None, FAR, 1 << 20, None) == p.VGG19_ERR_ARG


WS = FAR + (1 << 24)


@pytest.mark.parametrize("over,code", [
    (dict(loss=FAR + 2), "ARG"), (dict(lse=FAR + 4097), "ARG"), (dict(ws=None), "WORKSPACE"), (dict(ws=WS + 16), "WORKSPACE"), (dict(size=100), "WORKSPACE"),
    (dict(loss=FAR + 4096 + 16), "ARG"), (dict(loss=SOME), "ARG"), (dict(lse=SOME + (1 << 16) + 12796), "ARG"), (dict(loss=SOME + (2 << 16)), "ARG"), (dict(lse=SOME + (3 << 16) - 4), "ARG"),
    (dict(lse=WS), "ARG"), (dict(ws=SOME), "ARG")])
def test_the_loss_refuses(p, over, code):
    a = dict(loss=FAR, lse=FAR + 4096, ws=WS, size=1 << 30)
    a.update(over)
    assert p.binding.load().vgg19_linear_cross_entropy(ctypes.byref(layer(p)), *a.values(), None) == code_of(p, code) and p.vgg19_last_error()


@pytest.mark.parametrize("over,code", [
    (dict(lse=None), "ARG"), (dict(d_loss=None), "ARG"), (dict(lse=FAR + 2), "ARG"), (dict(d_loss=FAR + 1), "ARG"), (dict(lddx=63), "SHAPE"), (dict(lddw=63), "SHAPE"), (dict(lddx=1 << 36), "SHAPE"),
    (dict(dw_dtype=2), "ARG"), (dict(dx=FAR + 8193), "ARG"), (dict(dw=FAR + 65538, dw_dtype=0), "ARG"), (dict(db=FAR + (1 << 20) + 2), "ARG"), (dict(ws=None), "WORKSPACE"),
    (dict(ws=WS + 128), "WORKSPACE"), (dict(size=1000), "WORKSPACE"), (dict(dx=SOME), "ARG"), (dict(dw=SOME + (1 << 16)), "ARG"), (dict(dx=FAR + 65536), "ARG"), (dict(db=FAR), "ARG"),
    (dict(dx=FAR + 4096 - 126), "ARG"), (dict(db=SOME + (2 << 16)), "ARG"), (dict(dw=WS), "ARG"), (dict(ws=FAR + 65536), "ARG")])
def test_the_gradients_refuse(p, over, code):
    a = dict(lse=FAR, d_loss=FAR + 4096, dx=FAR + 8192, lddx=64, dw=FAR + 65536, dw_dtype=1, lddw=64, db=FAR + (1 << 20), ws=WS, size=1 << 30)
    a.update(over)
    assert p.binding.load().vgg19_linear_cross_entropy_backward(ctypes.byref(layer(p)), *a.values(), None) == code_of(p, code) and p.vgg19_last_error()


def test_nothing_asked_for_is_no_work(p):
    lib, some = p.binding.load(), layer(p)
    assert lib.vgg19_linear_cross_entropy(ctypes.byref(some), None, None, WS, 1 << 30, None) == p.VGG19_OK
    assert lib.vgg19_linear_cross_entropy(ctypes.byref(layer(p, rows=0, x=None, w=None, labels=None)), None, None, None, 0, None) == p.VGG19_OK
    assert lib.vgg19_linear_cross_entropy_backward(ctypes.byref(some), FAR, FAR + 4096, None, 0, None, 0, 0, None, WS, 1 << 30, None) == p.VGG19_OK
    assert lib.vgg19_dropout(None, 1, 0, 5, 5, 0.5, 1, 0, None, 0, None, 5, None) == p.VGG19_OK


def test_set_dropout_refuses_no_network(p):
    assert p.binding.load().vgg19_set_dropout(None, 0.5, 1, 0) == p.VGG19_ERR_ARG


def test_the_binding_refuses_what_does_not_fit(p):
    x, w = torch.zeros(2, 8), torch.zeros(5, 8)
    for call, code in [
            (lambda: p.vgg19_dropout(x, x, 0.5, 1), "ARG"), (lambda: p.vgg19_dropout(x[0], x, 0.5, 1), "SHAPE"), (lambda: p.vgg19_dropout(x.double(), x, 0.5, 1), "ARG"),
            (lambda: p.vgg19_dropout_backward(x, x, 0.5, 1), "ARG"), (lambda: p.vgg19_linear_cross_entropy(x, w, None, None, None, None, None), "ARG"),
            (lambda: p.vgg19_linear_cross_entropy_backward(x, w, None, None, None, None, None, None, None, None), "ARG"),
            (lambda: p.vgg19_linear_cross_entropy_bytes(x, w, True), "ARG")]:
        with pytest.raises(p.Vgg19Error) as e:
            call()
        assert e.value.code == code_of(p, code)


def test_workspaces_have_room_for_what_is_laid_out_anew(p):
    """x and w that copies cannot read where they lie, or that are fp32 (for more than eight rows), take more."""
    size = lambda back, **over: p.binding.load().vgg19_linear_cross_entropy_bytes(ctypes.byref(layer(p, rows=20, **over)), back)  # noqa: E731
    for back in (0, 1):
        plain = size(back)
        assert size(back, ldx=65) >= plain + 20 * 64 * 2 and size(back, ldw=65) >= plain + 100 * 64 * 2 and size(back, w=SOME + 2) >= plain + 100 * 64 * 2
        assert size(back, dtype=0) >= plain + 120 * 64 * 6
