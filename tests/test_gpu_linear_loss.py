"""The last dense layer with its softmax cross entropy against the formulas in 64 bits, value by value.

Tolerances, with u = 2^-24 (half a step of fp32) and h = 2^-8 (half a step of bf16), h = 0 for fp32 tensors:
  z     products of bf16 values are exact and so are an fp32 value's three terms; what is left out of an fp32 product is below 2^-23 of it.  A sum
        of n instructions, each adding 16 products to a sum so far below R (five standard deviations of the sum), loses at most a whole step of
        it each: n 2u R.  Then a bias is added: u |z|.
  lse   z's error, exponentials (2u each) and their sums (at most 32 + 4 terms and the parts in a row), a logarithm
  dz    d_loss p times z's and lse's errors and two of an exponential, roundings of d_loss p and of p - 1
  dx    dz's error times |w|, dz rounded to bf16 (h) times |w|, n instructions as above on sums below sum |dz w|, the result rounded (h or u)
  dw    the same with |x|;  db   dz's error, and a rounding for every addition on the way
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


def randn(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device=DEV) * std


def rows_of(gen, rows, cols, dtype, std=1.0, pad=0, skip=0):
    """Rows of a wider buffer, the first `skip` values into it."""
    return (randn(gen, rows, cols + pad + skip, std=std)).to(dtype)[:, skip:skip + cols]


class Case:
    def __init__(self, rows, inner, classes, dtype="bf16", seed=0, pad=0, skip=0, bias=True, std=2.0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype = TYPES[dtype]
        self.x = rows_of(g, rows, inner, self.dtype, pad=pad, skip=skip)
        self.w = rows_of(g, classes, inner, self.dtype, std=std / math.sqrt(inner), pad=pad, skip=skip)
        self.bias = randn(g, classes, std=0.3) if bias else None
        self.labels = torch.randint(0, classes, (rows,), generator=g, device=DEV, dtype=torch.int32)
        self.d_loss = randn(g, rows) / rows
        self.rows, self.inner, self.classes = rows, inner, classes

    def run(self, p, stream=None, dw_dtype=None, workspaces=None, out_pad=0, backward=True, check=True):
        st = stream or torch.cuda.current_stream()
        f32 = {"dtype": torch.float32, "device": DEV}
        nan = float("nan")
        self.loss, self.lse = torch.full((self.rows,), nan, **f32), torch.full((self.rows,), nan, **f32)
        ws = workspaces or [torch.empty(p.vgg19_linear_cross_entropy_bytes(self.x, self.w, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
        p.vgg19_linear_cross_entropy(self.x, self.w, self.bias, self.labels, self.loss, self.lse, ws[0], st)
        if backward:
            self.dx = torch.full((self.rows, self.inner + out_pad), nan, dtype=self.dtype, device=DEV)[:, :self.inner]
            self.dw = torch.full((self.classes, self.inner + out_pad), nan, dtype=dw_dtype or self.dtype, device=DEV)[:, :self.inner]
            self.db = torch.full((self.classes,), nan, **f32)
            p.vgg19_linear_cross_entropy_backward(self.x, self.w, self.bias, self.labels, self.lse, self.d_loss, self.dx, self.dw, self.db, ws[1], st)
        if check:
            p.vgg19_ops_status(st)
        return self

    def check(self, backward=True):
        x, w = self.x.double(), self.w.double()
        z = x @ w.T + (self.bias.double() if self.bias is not None else 0.0)
        real = (self.labels >= 0) & (self.labels < self.classes)
        at = self.labels.clamp(0, self.classes - 1).long()[:, None]
        lse = torch.logsumexp(z, 1)
        half = 2.0 ** -8 if self.dtype == torch.bfloat16 else U
        steps = self.inner / 16 + 2
        spread = (x.square() @ w.square().T).sqrt()  # of the sums behind z
        ez = steps * 2 * U * 5 * spread + 4 * U * spread * math.sqrt(self.inner) + U * z.abs().nan_to_num(0, 0, 0)
        e_lse = ez.amax(1) + (2 + 40 + self.classes / 1024 + 2) * 2 * U + 2 * U * lse.abs().nan_to_num(0, 0, 0)
        label_z = z.gather(1, at)[:, 0]
        loss = torch.where(real, lse - label_z, 0.0)
        self.near(self.lse, lse, e_lse, "lse")
        self.near(self.loss[real], loss[real], (e_lse + ez.amax(1) + 2 * U * loss.abs().nan_to_num(0, 0, 0))[real], "loss")
        assert (self.loss[self.labels == -1] == 0).all()
        if not backward:
            return
        g = torch.where(real & torch.isfinite(lse), self.d_loss.double(), 0.0)[:, None]
        prob = torch.exp(z - torch.where(torch.isfinite(lse), lse, math.inf)[:, None])
        one = torch.zeros_like(z).scatter_(1, at, 1.0)
        dz = g * (prob - one)
        edz = g.abs() * prob * (ez + e_lse[:, None] + 8 * U) + 2 * U * dz.abs()
        rounding = half if self.dtype == torch.bfloat16 else 2 * U
        def bound(e, d, other, n):
            size = d.abs() @ other.abs()
            return e @ other.abs() + rounding * size + (n / 16 + 2) * 2 * U * size
        dx, dw, db = dz @ w, dz.T @ x, dz.sum(0)
        self.near(self.dx, dx, bound(edz, dz, w, self.classes) + half * dx.abs(), "dx")
        out = 2.0 ** -8 if self.dw.dtype == torch.bfloat16 else U
        self.near(self.dw, dw, bound(edz.T, dz.T, x, self.rows) + out * dw.abs(), "dw")
        self.near(self.db, db, edz.sum(0) + (5 + self.rows / 32 + 2) * U * dz.abs().sum(0), "db")

    @staticmethod
    def near(got, want, tolerance, name):
        got = got.double()
        same = (got == want) | (got.isnan() & want.isnan())
        off = torch.where(same, 0.0, (got - want).abs() - tolerance)
        assert not off.isnan().any() and (off <= 1e-37).all(), (name, float(off.nan_to_num(1e9).max()), int((off > 0).sum()), off.numel())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,inner,classes", [
    (1, 1, 1), (1, 1, 2), (1, 64, 32), (2, 8, 3), (5, 7, 129), (31, 63, 127), (33, 65, 257), (100, 512, 1000), (127, 72, 255), (129, 1000, 513), (256, 64, 256),
    (257, 96, 511), (300, 333, 2049), (513, 200, 77), (1, 4096, 1000), (100, 4096, 1000), (3, 2500, 5003), (700, 48, 9001)])
def test_against_the_formulas(p, rows, inner, classes, dtype):
    Case(rows, inner, classes, dtype, seed=rows + inner).run(p).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7, 8, 9, 16, 23, 25])
@pytest.mark.parametrize("inner,classes,pad,skip", [(1, 5, 0, 0), (255, 100, 0, 0), (264, 1000, 0, 0), (4096, 300, 0, 0), (4097, 33, 3, 0), (8192, 90, 0, 0), (8200, 17, 0, 0), (100, 20011, 4, 0), (333, 2049, 3, 1),
                                                    (64, 9500, 8, 0)])
def test_a_few_rows(p, rows, inner, classes, pad, skip, dtype):
    """Up to eight rows, and up to 24 for the loss alone, have kernels of their own, up to 32768 / rows inputs."""
    Case(rows, inner, classes, dtype, seed=rows, pad=pad, skip=skip).run(p, dw_dtype=torch.float32 if classes == 33 else None).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,inner,classes,pad,skip,out_pad", [(40, 64, 300, 8, 0, 0), (40, 64, 300, 3, 0, 1), (40, 64, 300, 7, 1, 8), (70, 333, 130, 5, 0, 3), (1, 64, 40, 9, 1, 5),
                                                                   (6, 332, 1300, 0, 0, 0), (6, 332, 1300, 4, 0, 4), (6, 332, 1300, 3, 1, 3), (2, 332, 1300, 4, 4, 1)])
def test_rows_of_wider_buffers(p, rows, inner, classes, pad, skip, out_pad, dtype):
    c = Case(rows, inner, classes, dtype, pad=pad, skip=skip).run(p, out_pad=out_pad)
    c.check()
    for t in (c.dx, c.dw):  # what lies behind the rows is as it was
        whole = t.as_strided((t.shape[0], t.shape[1] + out_pad), (t.shape[1] + out_pad, 1)) if out_pad else t
        assert bool(whole[:, t.shape[1]:].isnan().all())


@pytest.mark.parametrize("bias", [True, False])
def test_gradients_of_weights_in_fp32(p, bias):
    Case(200, 130, 700, "bf16", bias=bias).run(p, dw_dtype=torch.float32).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_only_fill_the_batch_and_excluded_classes(p, dtype):
    c = Case(130, 100, 700, dtype)
    c.labels[::3] = -1
    excluded = torch.arange(0, 700, 7, device=DEV)
    c.bias[excluded] = -math.inf
    c.labels[c.labels % 7 == 0] = 1
    c.run(p).check()
    assert (c.dx[::3] == 0).all() and (c.dw[excluded] == 0).all() and (c.db[excluded] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_excluded_labels_and_rows_without_a_class(p, dtype):
    c = Case(70, 100, 300, dtype)
    c.bias[5] = -math.inf
    c.labels[:4] = 5
    c.run(p)
    assert torch.equal(c.loss == math.inf, c.labels == 5) and not c.loss.isnan().any()
    c.check()
    c.bias[:] = -math.inf
    c.run(p)
    assert (c.lse == -math.inf).all() and (c.loss == math.inf).all()
    assert (c.dx == 0).all() and (c.dw == 0).all() and (c.db == 0).all()
    c.bias[17] = 0.25  # one class left: certain
    c.labels[:] = 17
    c.run(p)
    assert (c.loss == 0).all() and (c.dx == 0).all() and (c.dw == 0).all()


def test_the_lowest_bias_is_a_number(p):
    c = Case(70, 100, 300)
    c.bias[::2] = torch.finfo(torch.float32).min
    c.labels[:] = 1 + 2 * (c.labels % 150)
    c.run(p)
    assert torch.isfinite(c.loss).all() and (c.dw[::2] == 0).all()
    c.bias[:] = -1e30
    c.labels[:] = 3
    c.run(p)
    assert torch.allclose(c.loss, torch.full_like(c.loss, math.log(300)), atol=1e-5) and torch.isfinite(c.dx).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_what_is_not_finite_stays_in_its_row(p, dtype):
    c = Case(300, 100, 300, dtype)
    c.x[7, 3], c.x[280, 99] = math.nan, math.nan
    c.bias[4] = math.nan
    c.run(p)
    assert c.lse.isnan().all()
    c.bias[4] = 0.0
    c.run(p)
    bad = torch.zeros(300, dtype=torch.bool, device=DEV)
    bad[[7, 280]] = True
    assert c.lse[bad].isnan().all() and c.loss[bad].isnan().all() and c.dx[bad].isnan().all()
    assert torch.isfinite(c.lse[~bad]).all() and torch.isfinite(c.loss[~bad]).all() and torch.isfinite(c.dx[~bad]).all()
    c.x[7, 3], c.x[280, 99] = 0.0, 0.0
    c.bias[4] = math.inf
    c.run(p)
    assert c.lse.isnan().all()


def test_rows_without_a_label_may_hold_anything_in_a_score(p):
    c = Case(64, 64, 100)
    good = Case(64, 64, 100).run(p, backward=False)
    c.labels[::2] = -1
    c.x[::2] = math.nan
    c.run(p, backward=False)
    assert (c.loss[::2] == 0).all() and torch.equal(c.loss[1::2], good.loss[1::2])


def test_labels_outside_the_classes_of_a_few_rows(p):
    c, st = Case(5, 64, 100, "fp32"), torch.cuda.current_stream()
    c.labels[:] = torch.tensor([100, 5, -2, -(1 << 31), 7], dtype=torch.int32, device=DEV)
    c.run(p, check=False)
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_ops_status(st)
    assert e.value.code == p.VGG19_ERR_ARG
    p.vgg19_ops_status(st)
    c.run(p, backward=False, check=False)
    with pytest.raises(p.Vgg19Error):
        p.vgg19_ops_status(st)
    c.check()
    assert c.loss[[0, 2, 3]].isnan().all() and (c.dx[[0, 2, 3]] == 0).all()


def test_labels_outside_the_classes_are_reported_and_count_for_nothing(p):
    c = Case(300, 64, 100)
    c.labels[::7] = torch.tensor([100, -2, 1 << 30], dtype=torch.int32, device=DEV).repeat(15)[:43]
    st = torch.cuda.current_stream()
    p.vgg19_ops_status(st)
    c.run(p, check=False)
    with pytest.raises(p.Vgg19Error) as e:
        p.vgg19_ops_status(st)
    assert e.value.code == p.VGG19_ERR_ARG and "label" in str(e.value)
    p.vgg19_ops_status(st)
    assert c.loss[::7].isnan().all() and (c.dx[::7] == 0).all()
    c.check()
    p.vgg19_linear_cross_entropy_backward(c.x, c.w, c.bias, c.labels, c.lse, c.d_loss, c.dx, None, None,
                                          torch.empty(p.vgg19_linear_cross_entropy_bytes(c.x, c.w, True), dtype=torch.uint8, device=DEV), st)
    with pytest.raises(p.Vgg19Error):
        p.vgg19_ops_status(st)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_each_result_alone_is_what_it_is_among_the_others(p, dtype):
    c = Case(200, 136, 500, dtype).run(p)
    ws = torch.empty(p.vgg19_linear_cross_entropy_bytes(c.x, c.w, True), dtype=torch.uint8, device=DEV)
    st = torch.cuda.current_stream()
    loss, lse = torch.empty_like(c.loss), torch.empty_like(c.lse)
    p.vgg19_linear_cross_entropy(c.x, c.w, c.bias, c.labels, loss, None, ws, st)
    p.vgg19_linear_cross_entropy(c.x, c.w, c.bias, c.labels, None, lse, ws, st)
    assert torch.equal(loss, c.loss) and torch.equal(lse, c.lse)
    for i in range(3):
        new = [torch.full_like(t, math.nan) if k == i else None for k, t in enumerate((c.dx, c.dw, c.db))]
        p.vgg19_linear_cross_entropy_backward(c.x, c.w, c.bias, c.labels, c.lse, c.d_loss, *new, ws, st)
        assert torch.equal(new[i], (c.dx, c.dw, c.db)[i])


def test_no_rows(p):
    x, w = torch.empty(0, 64, device=DEV), torch.randn(10, 64, device=DEV)
    labels, none = torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV)
    dw, db, ws = torch.ones(10, 72, device=DEV), torch.ones(10, device=DEV), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    p.vgg19_linear_cross_entropy(x, w, None, labels, none, none, ws)
    p.vgg19_linear_cross_entropy_backward(x, w, None, labels, none, none, torch.empty(0, 64, device=DEV), dw[:, :64], db, ws)
    torch.cuda.synchronize()
    assert (dw[:, :64] == 0).all() and (dw[:, 64:] == 1).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_gradient_against_differences(p, dtype):
    """Of sum(d_loss * loss) along random directions.  The step e moves z by about e: the difference's own error is e^2 / 6 of the third derivative
    (below 1 a row) and the losses' roundings, 4e-7 * 12, over e."""
    c = Case(50, 64, 200, "fp32", std=1.0)
    c.d_loss = torch.rand(50, device=DEV) + 0.5
    if dtype == "bf16":
        c.x, c.w, c.dtype = c.x.bfloat16(), c.w.bfloat16(), torch.bfloat16
    c.run(p)
    total = float(c.d_loss.double() @ c.loss.double())
    g = torch.Generator(device=DEV).manual_seed(5)
    for name in ("x", "w", "bias"):
        value, grad = getattr(c, name).float(), {"x": c.dx, "w": c.dw, "bias": c.db}[name].double()
        u = torch.randn(value.shape, generator=g, device=DEV)
        u = u / (u.norm(dim=-1, keepdim=True) if name == "x" else math.sqrt(64) if name == "w" else 1.0)
        e = 2.0 ** -6
        ends = []
        for s in (e, -e):
            moved = Case(50, 64, 200, "fp32")
            moved.x, moved.w, moved.bias, moved.labels = c.x.float(), c.w.float(), c.bias, c.labels
            setattr(moved, name, value + s * u)
            ends.append(float(c.d_loss.double() @ moved.run(p, backward=False).loss.double()))
        slope = (ends[0] - ends[1]) / (2 * e)
        want = float((grad * u.double()).sum())
        size = float((grad.abs() * u.double().abs()).sum())
        assert abs(slope - want) <= 75 * (e * e / 6) * 4 + 75 * 12 * 4e-7 / e + (2.0 ** -8 * 3 * size if dtype == "bf16" else 0), (name, slope, want, total)


def test_the_same_bits_every_time_and_in_any_company(p):
    a, b = Case(300, 264, 5000, seed=1).run(p), Case(300, 264, 5000, seed=1).run(p)
    for n in ("loss", "lse", "dx", "dw", "db"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n


@pytest.mark.parametrize("rows,inner,classes,dtype,pad", [(20000, 40, 9000, "bf16", 0), (12000, 37, 9001, "fp32", 0), (50, 9001, 30000, "bf16", 3)])
def test_pieces_of_the_classes(p, rows, inner, classes, dtype, pad):
    """More rows times classes than one piece of dz holds, or more weights to be laid out than one piece has room for: dx is added up over pieces."""
    c = Case(rows, inner, classes, dtype, std=1.0, pad=pad).run(p)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,inner,classes", [(128, 72, 40000), (100, 4096, 6000), (2300, 80, 2300), (640, 3000, 640), (256, 1030, 3000), (64, 40000, 30), (5000, 100, 4), (260, 64, 9600),
                                                (130, 4096, 2049), (130, 4096, 5000), (130, 4096, 12001), (520, 1000, 12001), (400, 4096, 2049), (2400, 333, 5000), (4000, 200, 5000)])
def test_tiles_of_every_shape(p, rows, inner, classes, dtype):
    """Sizes for which the plan takes pairs and single CTAs, wide and narrow tiles, cut sums and whole ones."""
    Case(rows, inner, classes, dtype, seed=7).run(p).check()


@pytest.mark.parametrize("dtype,dw_dtype", [("bf16", None), ("bf16", torch.float32), ("fp32", None)])
@pytest.mark.parametrize("rows,inner,classes,pad", [(4037, 35, 48, 0), (3000, 130, 10, 3), (4096, 1000, 70, 0), (513, 8, 1, 0), (2500, 333, 300, 1), (16384, 129, 257, 0)])
def test_many_rows_against_few_classes(p, rows, inner, classes, pad, dtype, dw_dtype):
    """dw has few tiles, each a long sum, which is cut into parts; alone it is what it is among the others."""
    c = Case(rows, inner, classes, dtype, seed=classes, pad=pad).run(p, dw_dtype=dw_dtype, out_pad=pad)
    c.check()
    dw, ws = torch.full_like(c.dw, math.nan), torch.empty(p.vgg19_linear_cross_entropy_bytes(c.x, c.w, True), dtype=torch.uint8, device=DEV)
    p.vgg19_linear_cross_entropy_backward(c.x, c.w, c.bias, c.labels, c.lse, c.d_loss, None, dw, None, ws, torch.cuda.current_stream())
    assert torch.equal(dw, c.dw)


@pytest.mark.parametrize("rows,inner,classes,dtype", [(100, 264, 1000, "bf16"), (4, 264, 1000, "fp32"), (300, 333, 2049, "bf16"), (200, 64, 500, "fp32")])
def test_recorded_and_replayed_with_other_inputs(p, rows, inner, classes, dtype):
    c = Case(rows, inner, classes, dtype)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ws = [torch.empty(p.vgg19_linear_cross_entropy_bytes(c.x, c.w, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
        c.run(p, st, workspaces=ws)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        c.run(p, torch.cuda.current_stream(), workspaces=ws, check=False)
    for seed in (3, 4):
        other = Case(rows, inner, classes, dtype, seed=seed)
        for n in ("x", "w", "bias", "labels", "d_loss"):
            getattr(c, n).copy_(getattr(other, n))
        graph.replay()
        torch.cuda.synchronize()
        c.check()
        other.run(p)
        for n in ("loss", "lse", "dx", "dw", "db"):
            assert torch.equal(getattr(c, n), getattr(other, n)), n


@pytest.mark.parametrize("dtype,rows", [("bf16", 100), ("fp32", 100), ("fp32", 3)])
def test_recorded_behind_copies_clears_and_another_stream(p, dtype, rows):
    """What a recorded call reads may come from any kind of node: a copy, a clear, a kernel of a stream that joins."""
    c, other = Case(rows, 136, 700, dtype), Case(rows, 136, 700, dtype, seed=9)
    side = torch.cuda.Stream()
    ws = [torch.empty(p.vgg19_linear_cross_entropy_bytes(c.x, c.w, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
    c.run(p, workspaces=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st = torch.cuda.current_stream()
        side.wait_stream(st)
        with torch.cuda.stream(side):
            torch.add(other.w, 0, out=c.w)
            c.d_loss.copy_(other.d_loss)
        c.bias.zero_()
        c.x.copy_(other.x)
        st.wait_stream(side)
        c.labels.copy_(other.labels)
        c.run(p, st, workspaces=ws, check=False)
    c.x.zero_(), c.w.zero_(), c.bias.fill_(3.0), c.labels.zero_()
    graph.replay()
    torch.cuda.synchronize()
    c.check()
    assert torch.equal(c.x, other.x) and torch.equal(c.w, other.w)


def test_two_streams_at_once(p):
    cases = [Case(500, 520, 3001, seed=1), Case(300, 100, 700, "fp32", seed=2)]
    want = [Case(500, 520, 3001, seed=1).run(p), Case(300, 100, 700, "fp32", seed=2).run(p)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                c.run(p, s, check=False)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        for n in ("loss", "lse", "dx", "dw", "db"):
            assert torch.equal(getattr(c, n), getattr(w, n)), n
    p.vgg19_ops_status(streams[0])


@pytest.mark.parametrize("rows,inner,classes,dtype", [(128, 17000, 130000, "bf16"), (140000, 16400, 40, "bf16")])
def test_offsets_beyond_32_bits(p, rows, inner, classes, dtype):
    """The last rows of x and w, 2^31 values in and more, against the formulas."""
    c = Case(1, 1, 1, dtype)
    g = torch.Generator(device=DEV).manual_seed(1)
    c.x = torch.empty(rows, inner, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    c.w = torch.empty(classes, inner, dtype=torch.bfloat16, device=DEV).normal_(0, 2.0 / math.sqrt(inner), generator=g)
    c.bias = torch.full((classes,), -math.inf, device=DEV)
    c.bias[-32:] = 0.0  # only the last classes count
    c.labels = torch.full((rows,), -1, dtype=torch.int32, device=DEV)
    c.labels[-20:] = classes - 3
    c.d_loss = torch.full((rows,), 0.05, device=DEV)
    c.rows, c.inner, c.classes = rows, inner, classes
    c.run(p)
    last = Case(1, 1, 1, dtype)
    last.x, last.w, last.bias, last.labels, last.d_loss = c.x[-20:], c.w[-32:], c.bias[-32:], c.labels[-20:] - (classes - 32), c.d_loss[-20:]
    last.rows, last.inner, last.classes = 20, inner, 32
    last.loss, last.lse, last.dx, last.dw, last.db = c.loss[-20:], c.lse[-20:], c.dx[-20:], c.dw[-32:], c.db[-32:]
    last.check()
    assert not c.dx[:-20].any() and not c.dw[:-32].any()


def test_from_several_threads(p):
    """Calls of other sizes from two threads, each with its stream and workspaces: the results of the same calls one after another."""
    import threading
    cases = [[Case(rows, inner, classes, dtype, seed=7) for rows, inner, classes, dtype in sizes] for sizes in (
        [(8, 4096, 300, "fp32"), (1, 8000, 40, "fp32"), (100, 264, 1000, "bf16")], [(8, 33, 300, "fp32"), (1, 100, 40, "fp32"), (300, 72, 500, "fp32")])]
    want = [[[getattr(c.run(p), n).clone() for n in ("loss", "lse", "dx", "dw", "db")] for c in of] for of in cases]
    torch.cuda.synchronize()
    failed = []
    def work(of, wanted):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for _ in range(20):
                    for c, w in zip(of, wanted):
                        c.run(p, st, check=False)
                        st.synchronize()
                        if not all(torch.equal(getattr(c, n), t) for n, t in zip(("loss", "lse", "dx", "dw", "db"), w)):
                            failed.append((c.rows, c.inner))
        except Exception as e:  # (told by the assertion below)
            failed.append(e)
    threads = [threading.Thread(target=work, args=a) for a in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
