"""Dropout against the generator's definition in Python integers, bit for bit: the mask is whole numbers, and what stays is one product rounded once."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


def philox(block, step, seed):
    """Philox 4x32-10 (Salmon et al. 2011): four words of one block."""
    m = 0xFFFFFFFF
    c, k = [block & m, block >> 32 & m, step & m, step >> 32 & m], [seed & m, seed >> 32 & m]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & m, (a >> 32) ^ c[3] ^ k[1], a & m]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    return c


def halves(first, n, step, seed):
    """The 16 bits of values first .. first + n - 1."""
    out = []
    for block in range(first // 8, (first + n + 7) // 8):
        for w in philox(block, step, seed):
            out += [w & 0xFFFF, w >> 16]
    return np.array(out[first % 8:first % 8 + n])


def expected(x, rate, seed, step=0, first=0):
    t = math.floor(float(np.float32(rate)) * 65536 + 0.5)
    keep = torch.from_numpy(halves(first, x.numel(), step, seed) >= t).to(DEV).view(x.shape)
    scale = np.float32(65536 / (65536 - t)) if t < 65536 else 0.0
    return torch.where(keep, x.float() * float(scale), 0.0).to(x.dtype)


def test_the_generator_gives_the_published_numbers():
    """Known answers of the generator's authors: counter and key of zeros, of ones, and of digits of pi."""
    words = lambda c, k: philox(c[0] | c[1] << 32, c[2] | c[3] << 32, k[0] | k[1] << 32)  # noqa: E731
    assert words([0] * 4, [0] * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert words([0xffffffff] * 4, [0xffffffff] * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert words([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0]) == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols,pad,skip", [(1, 1, 0, 0), (1, 7, 0, 0), (1, 8, 0, 0), (3, 5, 0, 0), (3, 5, 2, 0), (7, 64, 0, 0), (7, 64, 8, 0), (7, 64, 8, 8), (7, 64, 1, 0),
                                                (7, 64, 0, 1), (300, 1, 0, 0), (300, 1, 3, 0), (33, 257, 0, 0), (33, 257, 7, 0), (5, 1000, 24, 0), (2, 4096, 0, 0)])
def test_against_the_definition(p, rows, cols, pad, skip, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows * cols)
    wide = cols + pad
    x = torch.randn(rows * wide + skip, generator=g, device=DEV).to(TYPES[dtype])[skip:].view(rows, wide)[:, :cols]
    for rate, seed, step, first in ((0.5, 1, 0, 0), (0.1, (1 << 64) - 5, (1 << 63) + 9, 0), (0.9, 77, 3, 16), (0.3, 5, 1 << 40, 1000003), (0.25, 9, 1, (1 << 35) + 5)):
        out = torch.full((rows * wide + skip,), 3.0, dtype=TYPES[dtype], device=DEV)
        y = out[skip:].view(rows, wide)[:, :cols]
        p.vgg19_dropout(x, y, rate, seed, step, first=first)
        want = expected(x, rate, seed, step, first)
        assert torch.equal(y, want), (rate, first)
        assert (out[:skip] == 3).all() and (out[skip:].view(rows, wide)[:, cols:] == 3).all()
        dx = torch.empty(rows, cols, dtype=TYPES[dtype], device=DEV)
        p.vgg19_dropout_backward(x, dx, rate, seed, step, first=first)
        assert torch.equal(dx, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols,pad", [(64, 0), (64, 8), (37, 0), (37, 2)])
def test_in_place(p, cols, pad, dtype):
    x = torch.randn(50, cols + pad, device=DEV).to(TYPES[dtype])
    want = expected(x[:, :cols], 0.4, 3, 2)
    p.vgg19_dropout(x[:, :cols], x[:, :cols], 0.4, 3, 2)
    assert torch.equal(x[:, :cols], want)


@pytest.mark.parametrize("cols", [64, 63])
def test_rates_at_the_ends_and_in_between(p, cols):
    x = torch.randn(100, cols, device=DEV)
    for rate in (0.0, 1.0, 2.0 ** -16, 2.0 ** -18, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 1 / 3):
        y = torch.empty_like(x)
        p.vgg19_dropout(x, y, rate, 11)
        assert torch.equal(y, expected(x, rate, 11)), rate
    p.vgg19_dropout(x, y, 0.0, 11)
    assert torch.equal(x, y)


@pytest.mark.parametrize("cols", [64, 63])
def test_dropped_values_may_be_anything(p, cols):
    x = torch.full((64, cols), math.nan, device=DEV)
    y = torch.empty_like(x)
    p.vgg19_dropout(x, y, 1.0, 1)
    assert (y == 0).all()
    p.vgg19_dropout(x, y, 0.5, 1)
    assert torch.equal(y.isnan(), expected(torch.ones_like(x), 0.5, 1) != 0) and (y[~y.isnan()] == 0).all()


def test_a_mask_goes_by_place_alone(p):
    """The same for both types, for strided rows, and for shards that say where they begin."""
    ones = torch.ones(60, 40, device=DEV)
    whole = torch.empty_like(ones)
    p.vgg19_dropout(ones, whole, 0.5, 123, 4)
    half = torch.empty(60, 40, dtype=torch.bfloat16, device=DEV)
    p.vgg19_dropout(ones.bfloat16(), half, 0.5, 123, 4)
    assert torch.equal(half.float(), whole)
    for a, b in ((0, 13), (13, 60), (59, 60)):
        part = torch.empty(b - a, 40, device=DEV)
        p.vgg19_dropout(ones[a:b], part, 0.5, 123, 4, first=a * 40)
        assert torch.equal(part, whole[a:b])


def test_every_step_and_seed_has_a_mask_of_its_own_at_the_rate(p):
    """Masks of a million values: the share that stays is within five standard deviations of 1 - q, and two masks agree as often as independent ones do."""
    x = torch.ones(1000, 1000, device=DEV)
    masks = []
    for seed, step in ((1, 0), (1, 1), (2, 0), (1 << 32, 0), (1, 1 << 32)):
        y = torch.empty_like(x)
        p.vgg19_dropout(x, y, 0.3, seed, step)
        masks.append(y > 0)
        q = math.floor(0.3 * 65536 + 0.5) / 65536
        assert abs(float(masks[-1].double().mean()) - (1 - q)) < 5 * math.sqrt(q * (1 - q) / 1e6)
    same = 0.7 ** 2 + 0.3 ** 2
    for i in range(5):
        for j in range(i):
            assert abs(float((masks[i] == masks[j]).double().mean()) - same) < 5 * math.sqrt(same * (1 - same) / 1e6) + 1e-4


def test_recorded_with_a_counter_each_replay_has_another_mask(p):
    x = torch.randn(30, 64, device=DEV)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    counter = torch.zeros(1, dtype=torch.int64, device=DEV)
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    p.vgg19_dropout(x, y, 0.5, 9, 100, counter)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        p.vgg19_dropout(x, y, 0.5, 9, 100, counter, stream=torch.cuda.current_stream())
        p.vgg19_dropout_backward(x, dx, 0.5, 9, 100, counter, stream=torch.cuda.current_stream())
        counter += 1
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        want = expected(x, 0.5, 9, 100 + k)
        assert torch.equal(y, want) and torch.equal(dx, want)


def test_no_rows(p):
    x = torch.empty(0, 64, device=DEV)
    p.vgg19_dropout(x, torch.empty_like(x), 0.5, 1)
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(p):
    """The last values of more than 2^32, by vectors and by the general kernel."""
    n = (1 << 32) + 1000
    for cols in (1 << 16, 1000003):
        rows = n // cols + 1
        x = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
        p.vgg19_dropout(x, x, 0.5, 7, 1)
        tail = x[-1, -1000:]
        want = expected(torch.ones(1, 1000, device=DEV), 0.5, 7, 1, rows * cols - 1000)[0]
        assert torch.equal(tail.float(), want)
        del x, tail
    x = torch.ones(5000, 900001, dtype=torch.bfloat16, device=DEV)[:, :900000]
    p.vgg19_dropout(x, x, 0.5, 7, 1)
    assert torch.equal(x[-1, -1000:].float(), expected(torch.ones(1, 1000, device=DEV), 0.5, 7, 1, 5000 * 900000 - 1000)[0])
