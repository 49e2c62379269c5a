"""Workspace sizes of the last layer with its loss, and numbers that dropout takes, on the host alone, at the ends of what the library takes."""
import ctypes
import math
import random
import subprocess
import sys

import pytest

import __graft_entry__ as g

SOME = 1 << 20  # stands for a device address; nothing reads it


@pytest.fixture(scope="module")
def p():
    g.build()
    import paper_1810_09868_b200 as pkg
    return pkg


def size_of(p, rows, inner, classes, dtype, backward):
    layer = p.binding.vgg19_linear_loss(SOME, inner, SOME + (1 << 16), inner, None, SOME + (2 << 16), rows, inner, classes, dtype)
    return p.binding.load().vgg19_linear_cross_entropy_bytes(ctypes.byref(layer), backward)


def test_a_layer_of_no_rows_has_a_workspace(p):
    """In a process of its own, which a division by the number of rows would end."""
    ask = ("import sys; sys.path.insert(0, 'tests'); import paper_1810_09868_b200 as p; from test_head_sizes_cpu import size_of; "
           "print([size_of(p, 0, 64, 100, dtype, backward) for dtype in (p.VGG19_FP32, p.VGG19_BF16) for backward in (0, 1)])")
    done = subprocess.run([sys.executable, "-c", ask], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])
    assert done.stdout.split("\n")[-2] == str([256] * 4), done.stdout


@pytest.mark.parametrize("rows,inner,classes,dtype", [(32768, 128, 262144, 1), (65536, 64, 1 << 20, 1), (33216, 1, 1 << 20, 1), (20000, 17, 500000, 1), (32768, 128, 262144, 0), (8, 4096, 50021, 0),
                                                      (100, 4096, 1000, 1), (1, 1, 1, 0)])
def test_the_gradients_workspace_does_for_the_loss_too(p, rows, inner, classes, dtype):
    assert size_of(p, rows, inner, classes, dtype, 1) >= size_of(p, rows, inner, classes, dtype, 0) >= 256


def test_the_gradients_workspace_does_for_the_loss_at_any_size(p):
    rng = random.Random(7)

    def log(most):
        return int(math.exp(rng.uniform(0, math.log(most))))

    for _ in range(3000):
        rows, classes = log(1 << 22), log(1 << 24)
        if rows * classes <= 1 << 44:
            a = rows, log(1 << 20), classes, rng.randrange(2)
            assert size_of(p, *a, 1) >= size_of(p, *a, 0) > 0, a


def test_fewer_rows_may_take_more(p):
    """As the header says: a smaller batch is asked for by itself, and too small a workspace is refused before anything runs."""
    many, fewer = size_of(p, 1216, 4096, 1000, 1, 0), size_of(p, 1152, 4096, 1000, 1, 0)
    assert many < fewer
    layer = p.binding.vgg19_linear_loss(SOME, 4096, SOME + (1 << 24), 4096, None, SOME + (1 << 26), 1152, 4096, 1000, 1)
    far = 1 << 30
    assert p.binding.load().vgg19_linear_cross_entropy(ctypes.byref(layer), far, None, far + (1 << 20), many, None) == p.VGG19_ERR_WORKSPACE


@pytest.mark.parametrize("seed,first_pass", [(-1, 0), (1 << 64, 0), (0, -1), (0, 1 << 64), (0, (1 << 64) + 3)])
def test_a_networks_dropout_takes_no_number_modulo_2_to_the_64(p, seed, first_pass):
    """The C call's numbers have 64 bits: others are refused, as vgg19_dropout refuses them, not cut."""
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_set_dropout(None, 0.5, seed, first_pass)
    assert e.value.code == p.VGG19_ERR_ARG and "unsigned 64-bit" in str(e.value)


def test_a_dropouts_numbers_are_whole(p):
    for call in (lambda: p.vgg19_set_dropout(None, 0.5, 1.5), lambda: p.vgg19_set_dropout(None, 0.5, 1, 2.5)):
        with pytest.raises(p.Vgg19Error) as e:
            call()
        assert e.value.code == p.VGG19_ERR_ARG and "whole" in str(e.value)
