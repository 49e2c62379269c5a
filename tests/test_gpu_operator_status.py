"""What the operators report of waits that ran out, and to whom.  The waits are made to run out by the library's self-test: barriers that
expect one signal more than their copies give, over zeros, with a limit of about a millisecond.  Nothing faults: the kernels give up, end and return."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = ["VGG19_SELFTEST_DENSE_Q4", "VGG19_SELFTEST_UPDATE", "VGG19_SELFTEST_UPDATE_STEPS"]


@pytest.fixture(scope="module")
def p():
    import paper_1810_09868_b200 as pkg
    return pkg


def reported(p, fn, *a):
    """The code that a status call raises, or VGG19_OK."""
    try:
        fn(*a)
    except p.Vgg19Error as e:
        return e.code
    return p.VGG19_OK


def scratch(p):
    return torch.empty(p.VGG19_SELFTEST_BYTES, dtype=torch.uint8, device=DEV)


def calls(p, st):
    """One call of each operator; what they give."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    w, g, m = (torch.randn(96, 160, generator=gen, device=DEV) for _ in range(3))
    x, y = torch.randn(3, 160, generator=gen, device=DEV), torch.empty(3, 96, device=DEV)
    codes = torch.empty(p.vgg19_q4_code_bytes(96, 160), dtype=torch.uint8, device=DEV)
    scales = torch.empty(p.vgg19_q4_scale_bytes(96, 160, 64), dtype=torch.uint8, device=DEV)
    p.vgg19_q4_pack(w, 64, codes, scales, st)
    p.vgg19_q4_linear(x, codes, scales, 96, 64, y=y, stream=st)
    table = p.vgg19_muon_tensors([(w, None, g, m)])
    ws = torch.empty(p.vgg19_muon_workspace_bytes(table), dtype=torch.uint8, device=DEV)
    p.vgg19_muon_update(table, 0.1, 0.9, 0.0, 5, True, ws, st)
    return y, w, m


@pytest.mark.parametrize("kind", KINDS)
def test_a_wait_that_runs_out_is_reported_once(p, kind):
    st = torch.cuda.current_stream()
    before = calls(p, st)
    p.vgg19_ops_status(st)
    p.vgg19_selftest_operator_timeout(None, getattr(p, kind), scratch(p), st)
    assert reported(p, p.vgg19_ops_status, st) == p.VGG19_ERR_DEVICE_TIMEOUT
    p.vgg19_ops_status(st)
    for a, b in zip(before, calls(p, st)):  # and the operators work as they did
        assert torch.equal(a, b)
    p.vgg19_ops_status(st)


@pytest.mark.parametrize("kind", KINDS)
def test_what_runs_out_is_reported_to_its_owner_alone(p, kind):
    """Two networks that run 4-bit layers and the orthogonalised update, and calls without a handle beside them."""
    st, which, ws = torch.cuda.current_stream(), getattr(p, kind), scratch(p)
    nets = [p.Net(32, 32, 1, p.VGG19_BF16, seed=i, flags=p.VGG19_FLAG_DENSE_Q4) for i in (1, 2)]
    images = torch.rand(1, 32, 32, 3, device=DEV).to(torch.bfloat16)
    for net in nets:
        net.muon_step(torch.full((net.n_params,), 1e-3, device=DEV), torch.zeros(net.n_params, device=DEV), 1e-3)
    before = [net.forward(images).clone() for net in nets]
    status = [nets[0].sync_status, nets[1].sync_status, lambda: p.vgg19_ops_status(st)]
    for owner, handle in enumerate((nets[0].handle, nets[1].handle, None)):
        p.vgg19_selftest_operator_timeout(handle, which, ws, st)
        for other in {0, 1, 2} - {owner}:
            assert reported(p, status[other]) == p.VGG19_OK, (owner, other)
        assert reported(p, status[owner]) == p.VGG19_ERR_DEVICE_TIMEOUT
        assert [reported(p, s) for s in status] == [p.VGG19_OK] * 3
    for net, logits in zip(nets, before):
        assert torch.equal(net.forward(images), logits)
        net.sync_status()
        net.close()


def test_one_status_reports_all_that_was_recorded(p):
    """A bad id, a 4-bit layer's wait and an update's: the first status names them all, the next one finds none."""
    st, ws = torch.cuda.current_stream(), scratch(p)
    z, ids = torch.zeros(1, 10, device=DEV), torch.full((1, 1), 10, dtype=torch.int32, device=DEV)

    def bad_id():
        p.vgg19_logprobs(z, ids, torch.empty(1, 1, device=DEV), stream=st)

    for record, code, words in (
            ([bad_id], p.VGG19_ERR_ARG, ["id"]),
            ([bad_id, p.VGG19_SELFTEST_DENSE_Q4], p.VGG19_ERR_DEVICE_TIMEOUT, ["4-bit", "id"]),
            ([p.VGG19_SELFTEST_UPDATE, bad_id], p.VGG19_ERR_DEVICE_TIMEOUT, ["update", "id"]),
            ([p.VGG19_SELFTEST_DENSE_Q4, p.VGG19_SELFTEST_UPDATE], p.VGG19_ERR_DEVICE_TIMEOUT, ["4-bit", "update"])):
        for r in record:
            r() if callable(r) else p.vgg19_selftest_operator_timeout(None, r, ws, st)
        with pytest.raises(p.Vgg19Error) as e:
            p.vgg19_ops_status(st)
        assert e.value.code == code and all(w in str(e.value) for w in words), str(e.value)
        p.vgg19_ops_status(st)


def test_a_status_waits_for_its_own_stream_alone(p):
    """It is read while the legacy default stream is busy: the exchange runs on the stream that is asked about."""
    mine, other = torch.cuda.Stream(), torch.cuda.default_stream()
    net = p.Net(32, 32, 1, p.VGG19_BF16, seed=1, mode=p.VGG19_MODE_FORWARD)
    p.vgg19_ops_status(mine), net.sync_status(mine)
    done = torch.cuda.Event()
    with torch.cuda.stream(other):
        torch.cuda._sleep(2_000_000_000)  # about a second
        done.record()
    p.vgg19_ops_status(mine), net.sync_status(mine)
    assert not done.query()
    net.close()
    torch.cuda.synchronize()


def test_statuses_of_two_threads_do_not_wait_for_one_another(p):
    import threading
    busy, idle, done = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.Event()
    p.vgg19_ops_status(idle)
    with torch.cuda.stream(busy):
        torch.cuda._sleep(2_000_000_000)  # about a second
        done.record()
    started = threading.Event()
    other = threading.Thread(target=lambda: (started.set(), p.vgg19_ops_status(busy)))
    other.start()
    started.wait()
    other.join(0.05)  # it is in its call by now, waiting for its stream
    p.vgg19_ops_status(idle)
    assert other.is_alive() and not done.query()
    other.join()
