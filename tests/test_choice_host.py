"""Refusals of the draws and their loss: the entry points check their arguments before anything is
enqueued (no GPU needed)."""

import ctypes as C

import pytest

from paper_2608_27612_amd import emr


def call(scores=None, draws=1, u=64, index=64, **rule):
    s = emr.emr_scores(64, emr.EMR_F32, 2, 10, 10) if scores is None else scores
    r = emr.emr_sampling(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    for k, v in rule.items():
        setattr(r, k, v)
    return emr.lib().emr_sample(C.byref(s), C.byref(r), u, draws, index, None, None)


def loss(scores=None, temperature=1.0, index=64, out=64, grad=64, stride=10):
    s = emr.emr_scores(64, emr.EMR_F32, 2, 10, 10) if scores is None else scores
    return emr.lib().emr_answer_loss(C.byref(s), index, None, C.c_float(temperature), out, grad, stride,
                                     None)


BAD_SCORES = [(0, emr.EMR_F32, 2, 10, 10), (64, 3, 2, 10, 10), (64, -1, 2, 10, 10),
              (64, emr.EMR_F32, -1, 10, 10), (64, emr.EMR_F32, 2, 0, 10), (64, emr.EMR_F32, 2, 10, -1),
              (66, emr.EMR_F32, 2, 10, 10), (65, emr.EMR_F16, 2, 10, 10),
              (64, emr.EMR_F32, 2, 10, 1 << 61)]


@pytest.mark.parametrize("bad", BAD_SCORES)
def test_bad_scores(bad):
    for f in (call, loss):
        assert f(emr.emr_scores(*bad)) == emr.EMR_E_INVAL
        assert emr.lib().emr_last_error()


def test_too_many_rows_or_scores():
    for rows, n in ((1 << 31, 10), (2, 1 << 31)):
        for f in (call, loss):
            assert f(emr.emr_scores(64, emr.EMR_F32, rows, n, 0)) == emr.EMR_E_LIMIT


@pytest.mark.parametrize("rule", [
    dict(temperature=-0.5), dict(temperature=float("nan")), dict(top_k=-1), dict(top_p=0.0),
    dict(top_p=1.5), dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1),
    dict(min_p=float("nan"))])
def test_bad_rules(rule):
    assert call(**rule) == emr.EMR_E_INVAL
    name = next(iter(rule))
    assert name.encode() in emr.lib().emr_last_error()


def test_bad_buffers():
    assert call(draws=-1) == emr.EMR_E_INVAL
    assert call(draws=1 << 62) == emr.EMR_E_INVAL
    assert call(u=None) == emr.EMR_E_INVAL
    assert call(index=None) == emr.EMR_E_INVAL
    assert emr.lib().emr_sample(None, None, 64, 1, 64, None, None) == emr.EMR_E_INVAL
    s = emr.emr_scores(64, emr.EMR_F32, 2, 10, 10)
    assert emr.lib().emr_sample(C.byref(s), None, 64, 1, 64, None, None) == emr.EMR_E_INVAL
    assert call(draws=0) == emr.EMR_OK
    assert call(emr.emr_scores(None, emr.EMR_F32, 0, 10, 10)) == emr.EMR_OK


def test_bad_losses():
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-45):
        assert loss(temperature=t) == emr.EMR_E_INVAL
    assert loss(out=None, grad=None) == emr.EMR_E_INVAL
    assert loss(stride=9) == emr.EMR_E_INVAL
    assert loss(grad=66) == emr.EMR_E_INVAL
    assert loss(index=None) == emr.EMR_E_INVAL
    assert loss(emr.emr_scores(None, emr.EMR_F32, 0, 10, 10)) == emr.EMR_OK


def test_binding_refuses():
    torch = pytest.importorskip("torch")
    x = torch.zeros((2, 3))
    with pytest.raises(ValueError):
        emr.emr_sample(x, torch.zeros((2, 1)))
    with pytest.raises(ValueError):
        emr.emr_answer_loss(x, torch.zeros(2, dtype=torch.int32))


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_tensors_of_another_device_are_refused(monkeypatch):
    """A call launches on the current device (a stream's own): tensors that lie elsewhere would be read
    across, or not at all. (Tensors without memory stand for a second device's.)"""
    torch = pytest.importorskip("torch")
    from torch._subclasses.fake_tensor import FakeTensorMode

    class On:
        raw, device = None, 0

        def __init__(self, stream):
            pass

        def __enter__(self):
            return self

        def __exit__(self, *e):
            pass

    monkeypatch.setattr(emr, "_On", On)
    net = emr.Networks(None)
    net._counts = (2, 8, 5, 3, 1)  # genomes, nodes, edges, inputs, outputs
    with FakeTensorMode():
        def new(*shape, dtype=torch.float32, device="cuda:0"):
            return torch.empty(shape, dtype=dtype, device=device)

        def each(call, *tensors):
            for k in range(len(tensors)):
                for device in ("cuda:1", "cpu"):
                    args = list(tensors)
                    args[k] = torch.empty_like(args[k], device=device)
                    with pytest.raises(ValueError, match="device"):
                        call(*args)

        i32, u8 = torch.int32, torch.uint8
        each(lambda x, u: emr.emr_sample(x, u), new(4, 9), new(4, 2))
        each(lambda t, k, p, m: emr.emr_sample(new(4, 9), new(4, 2), t, k, p, m), new(4), new(4, dtype=i32), new(4),
             new(4))
        each(lambda x, i, s: emr.emr_answer_loss(x, i, s), new(4, 9), new(4, dtype=i32), new(4))
        each(net.set_weights, new(5))
        each(lambda x: net.activate_keep(x, 2), new(4, 3))
        each(lambda x, o, c, g: net.activate_backward(x, 2, o, emr.Kept(c, 4), g), new(4, 3), new(2, 4, 1),
             new(1, 1, 8, 4, dtype=u8), new(2, 4, 1))
        each(lambda c: emr.Kept(c, 4).values(), new(1, 1, 8, 4, dtype=u8))
