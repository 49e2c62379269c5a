"""Dropout and the last layer with its loss where calls meet one another, and at the ends of what they take."""
import math

import pytest
import torch

import seeded_inputs as si

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


@pytest.mark.parametrize("graph", [True, False])
def test_a_pass_right_behind_set_dropout_takes_its_masks(p, graph):
    """On a stream that is not ordered behind the library's own copies: the masks, logits and gradients of a pass that waited for everything."""
    B = 3
    images, labels = torch.from_numpy(si.images(B, 32, 32, seed=1)).to(DEV).bfloat16(), torch.from_numpy(si.labels(B, seed=2)).to(DEV)
    net = p.Net(32, 32, B, p.VGG19_BF16, seed=1, flags=0 if graph else p.VGG19_FLAG_NO_GRAPH)
    logits = torch.empty(B, 1000, device=DEV)
    ones = torch.ones(B, 4096, device=DEV, dtype=torch.bfloat16)
    kept = torch.empty_like(ones)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for k in range(12):
            got = []
            for wait in (True, False):
                net.set_dropout(0.5, seed=7, first_pass=3)  # (another state in between)
                net.backward(images, labels, logits=logits)
                net.set_dropout(0.25, seed=100 + k, first_pass=5 * k)
                if wait:
                    torch.cuda.synchronize()
                for _ in range(2):  # the second pass counts on from the first
                    grads, _ = net.backward(images, labels, logits=logits)
                    got.append((logits.clone(), grads.clone()))
                act = net.saved_tensor(B, p.VGG19_MODE_BACKWARD, 21).reshape(B, -1)
                p.vgg19_dropout(ones, kept, 0.25, 100 + k, 2 * (5 * k + 1), stream=st)
                assert (act[kept == 0] == 0).all() and (act[kept != 0] != 0).any()
            for i in (0, 1):
                assert torch.equal(got[i][0], got[2 + i][0]) and torch.equal(got[i][1], got[2 + i][1])
            assert not torch.equal(got[0][0], got[1][0])
    net.sync_status(st)
    net.close()


class Rows:
    """Inputs, results and a workspace of one call of the last layer with its loss."""

    def __init__(self, p, rows, inner, classes, dtype=torch.float32, seed=0, dw_dtype=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.p = p
        self.x = torch.randn(rows, inner, generator=g, device=DEV).to(dtype)
        self.w = (torch.randn(classes, inner, generator=g, device=DEV) * 2 / math.sqrt(inner)).to(dtype)
        self.bias = torch.randn(classes, generator=g, device=DEV) * 0.3
        self.labels = torch.randint(0, classes, (rows,), generator=g, device=DEV, dtype=torch.int32)
        self.d_loss = torch.randn(rows, generator=g, device=DEV)
        self.loss, self.lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        self.dx, self.db = torch.empty_like(self.x), torch.empty(classes, device=DEV)
        self.dw = torch.empty(classes, inner, dtype=dw_dtype or dtype, device=DEV)
        self.ws = torch.empty(max(p.vgg19_linear_cross_entropy_bytes(self.x, self.w, b) for b in (False, True)), dtype=torch.uint8, device=DEV)

    def forward(self, st):
        self.p.vgg19_linear_cross_entropy(self.x, self.w, self.bias, self.labels, self.loss, self.lse, self.ws, st)
        return self.loss, self.lse

    def backward(self, st):
        self.p.vgg19_linear_cross_entropy_backward(self.x, self.w, self.bias, self.labels, self.lse, self.d_loss, self.dx, self.dw, self.db, self.ws, st)
        return self.dx, self.dw, self.db


@pytest.mark.parametrize("rows,inner,classes", [(1, 64, 600), (2, 1000, 90), (4, 4096, 300), (7, 130, 5003), (8, 300, 40), (20, 264, 1000)])
def test_calls_back_to_back_on_one_workspace(p, rows, inner, classes):
    """Launches are set up while the ones before them run: every call reads what its own launches wrote to the workspace, not a line of the call before."""
    c = Rows(p, rows, inner, classes)
    st = torch.cuda.current_stream()
    scales = [1.0, -3.0, 0.25, 7.0]
    d_loss = [c.d_loss * s for s in scales]
    out = [[torch.empty_like(t) for t in (c.dx, c.dw, c.db)] for _ in scales]
    c.forward(st)
    alone = []
    for d in d_loss:
        torch.cuda.synchronize()
        c.d_loss = d
        alone.append([t.clone() for t in c.backward(st)])
        torch.cuda.synchronize()
    for _ in range(10):
        for d, (dx, dw, db) in zip(d_loss, out):  # nothing between the calls
            p.vgg19_linear_cross_entropy_backward(c.x, c.w, c.bias, c.labels, c.lse, d, dx, dw, db, c.ws, st)
        torch.cuda.synchronize()
        for got, want in zip(out, alone):
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows,inner,classes", [(1, 4096, 300), (8, 512, 1000), (24, 512, 700), (40, 264, 500)])
def test_weights_that_an_update_writes_right_before(p, rows, inner, classes):
    """An update's last kernel lets the next one in the stream be set up while it writes the weights; the loss behind it reads the new ones."""
    c, st = Rows(p, rows, inner, classes), torch.cuda.current_stream()
    grad, momentum = torch.randn_like(c.w), torch.zeros_like(c.w)
    table = p.vgg19_muon_tensors([(c.w, None, grad, momentum)])
    ws = torch.empty(p.vgg19_muon_workspace_bytes(table), dtype=torch.uint8, device=DEV)
    for _ in range(10):
        p.vgg19_muon_update(table, 0.5, 0.9, 0.0, 5, True, ws, stream=st)
        got = [t.clone() for t in c.forward(st)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, c.forward(st)))
        torch.cuda.synchronize()
    p.vgg19_ops_status(st)


@pytest.mark.parametrize("rows,classes", [(40, 300), (300, 300), (300, 1001), (1000, 40), (129, 8193)])
def test_infinities_leave_what_the_formula_leaves(p, rows, classes):
    """bf16 rows with an infinity whose products have one sign: z is -inf in every class of the row, which is then left none, wherever the tiles end."""
    inner = 72
    g = torch.Generator(device=DEV).manual_seed(rows + classes)
    x = torch.randn(rows, inner, generator=g, device=DEV).bfloat16()
    w = (torch.randn(classes, inner, generator=g, device=DEV) / 8).bfloat16()
    w[:, 5] = w[:, 5].abs() + 0.125
    x[::3, 5] = -math.inf
    labels = torch.randint(0, classes, (rows,), generator=g, device=DEV, dtype=torch.int32)
    loss, lse, d_loss = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.ones(rows, device=DEV)
    dx, db = torch.full_like(x, math.nan), torch.full((classes,), math.nan, device=DEV)
    st = torch.cuda.current_stream()
    ws = [torch.empty(p.vgg19_linear_cross_entropy_bytes(x, w, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
    p.vgg19_linear_cross_entropy(x, w, None, labels, loss, lse, ws[0], st)
    none = torch.zeros(rows, dtype=torch.bool, device=DEV)
    none[::3] = True
    assert (lse[none] == -math.inf).all() and (loss[none] == math.inf).all()
    assert torch.isfinite(lse[~none]).all() and torch.isfinite(loss[~none]).all()
    p.vgg19_linear_cross_entropy_backward(x, w, None, labels, lse, d_loss, dx, None, db, ws[1], st)
    p.vgg19_ops_status(st)
    assert (dx[none] == 0).all() and torch.isfinite(dx).all() and torch.isfinite(db).all()


@pytest.mark.parametrize("dw_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,inner,classes", [(200001, 4096, 1000), (300000, 1000, 4000), (1200000, 256, 9000), (1200000, 70, 300), (1 << 22, 64, 300)])
def test_sums_over_many_rows_do_not_drift(p, rows, inner, classes, dw_dtype):
    """dw of bf16 operands, all of one sign.  With w 0, no bias and an lse of 0, dz is exactly d_loss = 1 (0 at the label, class 0), so dw is
    x's column sums.  A tensor core's sum of at most 4096 products (32768 where the result is bf16), 256 instructions (2048) that may each lose a whole step of
    the sum so far, is within 256 2^-23 of its own; the sums of those are added in fp32, half a step 2^-24 each and one more for each of up to 64 parts; and
    a bf16 result is rounded."""
    f32 = dw_dtype == torch.float32
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = torch.empty(rows, inner, dtype=torch.bfloat16, device=DEV).uniform_(0.5, 1.0, generator=g)
    w, labels = torch.zeros(classes, inner, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    lse, d_loss = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    dw, db = torch.full((classes, inner), math.nan, device=DEV, dtype=dw_dtype), torch.full((classes,), math.nan, device=DEV)
    ws = torch.empty(p.vgg19_linear_cross_entropy_bytes(x, w, True), dtype=torch.uint8, device=DEV)
    st = torch.cuda.current_stream()
    p.vgg19_linear_cross_entropy_backward(x, w, None, labels, lse, d_loss, None, dw, db, ws, st)
    p.vgg19_ops_status(st)
    want = torch.zeros(inner, dtype=torch.float64, device=DEV)
    for a in range(0, rows, 50000):
        want += x[a:a + 50000].double().sum(0)
    off = max(((dw[a:a + 1000].double() - want).abs() / want).max().item() for a in range(1, classes, 1000))
    chain = (256 if f32 else 2048) * 2.0 ** -23 + (rows / 4096 + 66) * 2.0 ** -24
    assert not dw[0].any() and off <= chain + (0 if f32 else 2.0 ** -8), off
    assert db[0] == 0 and (db[1:] == rows).all()  # (whole numbers below 2^24)


@pytest.mark.parametrize("rows,inner,classes", [(100, 4096, 200000), (130, 1000, 700001), (2048, 4096, 70001), (3000, 3001, 40000), (1, 64, 1 << 24)])
def test_sums_over_many_classes_do_not_drift(p, rows, inner, classes):
    """dx of bf16 operands in the same way: x is 0, so that dz is d_loss = 1 everywhere but at the label, and dx is w's column sums, rounded to bf16."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = torch.zeros(rows, inner, dtype=torch.bfloat16, device=DEV)
    w = torch.empty(classes, inner, dtype=torch.bfloat16, device=DEV).uniform_(0.5, 1.0, generator=g)
    labels, lse, d_loss = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    dx, dw = torch.full_like(x, math.nan), torch.full_like(w, math.nan)
    ws = torch.empty(p.vgg19_linear_cross_entropy_bytes(x, w, True), dtype=torch.uint8, device=DEV)
    st = torch.cuda.current_stream()
    p.vgg19_linear_cross_entropy_backward(x, w, None, labels, lse, d_loss, dx, dw, None, ws, st)
    p.vgg19_ops_status(st)
    want = torch.zeros(inner, dtype=torch.float64, device=DEV)
    for a in range(1, classes, 50000):
        want += w[a:a + 50000].double().sum(0)
    off = ((dx.double() - want).abs() / want).max().item()
    assert off <= 2.0 ** -8 + 2048 * 2.0 ** -23 + (classes / 4096 + 66) * 2.0 ** -24 and not dw.any(), off


def test_a_description_counts_the_random_masks(p):
    net = p.Net(32, 32, 1, p.VGG19_BF16, seed=1, mode=p.VGG19_MODE_FORWARD)
    assert " rng=0\n" in p.vgg19_describe(net.handle)
    net.set_dropout(0.25)
    text = p.vgg19_describe(net.handle)
    assert "dropout at 0.25" in text and " rng=2 " in text and "rng=0" not in text
    net.set_dropout(0.0)
    assert " rng=0\n" in p.vgg19_describe(net.handle)
    net.close()


def test_one_status_names_all_kinds_at_once(p):
    """Words of five files: a bad id, bad labels of tiles and of a few rows, and the waits of all operators; the next status finds none."""
    st = torch.cuda.current_stream()
    p.vgg19_ops_status(st)
    ws = torch.empty(p.VGG19_SELFTEST_BYTES, dtype=torch.uint8, device=DEV)
    tiles, few = Rows(p, 40, 64, 300), Rows(p, 3, 64, 300)

    def bad_label(c):
        c.labels[-1] = 300
        c.forward(st)

    def bad_id():
        p.vgg19_logprobs(torch.zeros(1, 10, device=DEV), torch.full((1, 1), 10, dtype=torch.int32, device=DEV), torch.empty(1, 1, device=DEV), stream=st)

    wait = lambda kind: p.vgg19_selftest_operator_timeout(None, getattr(p, "VGG19_SELFTEST_" + kind), ws, st)  # noqa: E731
    kinds = {"4-bit": lambda: wait("DENSE_Q4"), "update": lambda: wait("UPDATE"), "with its loss": lambda: wait("LOSS"), "id outside": bad_id,
             "label outside": lambda: bad_label(tiles), "label": lambda: bad_label(few)}
    for chosen in [[k] for k in kinds] + [list(kinds), ["update", "label"], ["with its loss", "id outside"]]:
        for k in chosen:
            kinds[k]()
        with pytest.raises(p.Vgg19Error) as e:
            p.vgg19_ops_status(st)
        assert all(k in str(e.value) for k in chosen), str(e.value)
        assert e.value.code == (p.VGG19_ERR_DEVICE_TIMEOUT if {"4-bit", "update", "with its loss"} & set(chosen) else p.VGG19_ERR_ARG)
        p.vgg19_ops_status(st)


def test_a_status_of_all_operators_takes_about_as_long_as_a_networks(p):
    """One exchange on the device and one copy, whatever the number of words: it was six of each, six times a network's."""
    import time
    net = p.Net(32, 32, 1, p.VGG19_BF16, seed=1, mode=p.VGG19_MODE_FORWARD)
    st = torch.cuda.current_stream()

    def median(call):
        times = []
        for _ in range(300):
            a = time.perf_counter()
            call()
            times.append(time.perf_counter() - a)
        return sorted(times)[150]

    median(lambda: p.vgg19_ops_status(st)), median(lambda: net.sync_status(st))
    ratio = min(median(lambda: p.vgg19_ops_status(st)) / median(lambda: net.sync_status(st)) for _ in range(5))
    net.close()
    assert ratio < 3, ratio


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,inner,classes", [(7, 300, 500), (20, 512, 700), (100, 264, 1000), (300, 136, 2049), (2000, 40, 9001)])
def test_a_rows_results_do_not_depend_on_its_company(p, rows, inner, classes, dtype):
    """The same bits whatever the other rows hold, not-a-numbers and rows without a label among them."""
    c, st = Rows(p, rows, inner, classes, dtype), torch.cuda.current_stream()
    kept = torch.arange(0, rows, 3, device=DEV)
    others = torch.ones(rows, dtype=torch.bool, device=DEV)
    others[kept] = False
    c.forward(st)
    first = [t[kept].clone() for t in (c.loss, c.lse, c.backward(st)[0])]
    for fill in (0.0, 5.0, math.nan, math.inf):
        c.x[others] = fill
        c.labels[others] = -1 if fill != 5.0 else 0
        c.forward(st)
        assert all(torch.equal(a, b) for a, b in zip(first, (c.loss[kept], c.lse[kept], c.backward(st)[0][kept]))), fill
    p.vgg19_ops_status(st)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,classes", [(30, 100), (300, 700), (3000, 5000)])
def test_long_rows_of_one_sign_do_not_drift(p, rows, classes, dtype):
    """z of 65536 products of one sign.  A chain of 1024 of them is 64 instructions (for fp32 512 products, 32), each losing less than a step, 2^-23, of the
    sum so far (fp32: its five lesser products too, 2^-7 of that); 64 (128) chains are added, half a step each; then lse's own: within 2^-24 of its size and
    20 steps of an exponential sum's.  Terms that an fp32 product leaves out are below 3 2^-24 of it."""
    g = torch.Generator(device=DEV).manual_seed(classes)
    inner = 65536
    x, w = (torch.empty(n, inner, device=DEV).uniform_(0.5, 1.0, generator=g).to(dtype) for n in (rows, classes))
    labels, loss, lse = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    st = torch.cuda.current_stream()
    ws = torch.empty(p.vgg19_linear_cross_entropy_bytes(x, w, False), dtype=torch.uint8, device=DEV)
    p.vgg19_linear_cross_entropy(x, w, None, labels, loss, lse, ws, st)
    p.vgg19_ops_status(st)
    z = x.double() @ w.double().T
    want = torch.logsumexp(z, 1)
    relative = (64 + 64 / 2 if dtype == torch.bfloat16 else 32 * (1 + 2.0 ** -7) + 128 / 2 + 1.5) * 2.0 ** -23
    off = ((lse.double() - want).abs() - 20 * 2.0 ** -23).div(want.abs()).max().item()
    assert off <= relative + 2.0 ** -24, (off, relative)
