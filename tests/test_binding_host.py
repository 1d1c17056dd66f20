"""What the binding keeps and hands over, without a GPU: stand-ins for device tensors, and library calls that record instead of running."""
import copy
import os
import pickle

import numpy as np
import pytest

from paper_2003_10579_amd import ssgd


class Tensor:
    """As much of a device tensor as the binding looks at; its memory moves when it is copied."""
    is_cuda, device = True, "a GPU"

    def __init__(self, array):
        self.array = array

    shape = property(lambda self: self.array.shape)

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.array.itemsize

    def data_ptr(self):
        return self.array.ctypes.data


@pytest.fixture(scope="module")
def library():
    if not os.path.exists(ssgd._LIB_PATH):
        from paper_2003_10579_amd import build
        build.build()
    return ssgd.lib()


@pytest.fixture
def fresh(library, monkeypatch):
    """The binding as a new process has it, with a device that needs no starting."""
    import torch
    monkeypatch.setattr(torch.cuda, "init", lambda: None)
    for name in ("_torch", "_raw_stream", "_device_now", "_lib"):
        monkeypatch.setattr(ssgd, name, None)
    monkeypatch.setattr(ssgd, "_DTYPES", {})
    return torch


def _stored(rows=3, cols=40):
    return ssgd.MxTensor(Tensor(np.zeros((rows, 64), np.uint8)), Tensor(np.zeros((rows, 4), np.uint8)), "fp4", (rows, cols))


def test_a_stored_matrix_is_enough_to_begin_with(fresh):
    """The first thing that a program does may be a product of matrices that it has read from a file."""
    _stored()
    assert ssgd._torch is fresh and ssgd._lib is not None
    assert ssgd._DTYPES == {fresh.float32: ssgd.F32, fresh.bfloat16: ssgd.BF16}
    assert callable(ssgd._raw_stream) and callable(ssgd._device_now)


def test_arrays_that_are_no_matrix_are_refused_without_a_gpu(monkeypatch):
    monkeypatch.setattr(ssgd, "_torch", None)
    for values, scales, fmt, shape in ((np.zeros((3, 64), np.uint8), np.zeros((3, 3), np.uint8), "fp4", (3, 40)), (np.zeros((3, 64), np.uint8), np.zeros((3, 4), np.uint8), "fp6", (3, 40))):
        with pytest.raises(ssgd.SsgdError) as e:
            ssgd.MxTensor(Tensor(values), Tensor(scales), fmt, shape)
        assert e.value.status == ssgd.EINVAL
    assert ssgd._torch is None


def test_a_copied_matrix_has_its_own_addresses(fresh):
    """Copies, and what is read back from a pickle, point at their own arrays and not where the first ones were."""
    q = _stored()
    q.values.array[:], q.scales.array[:] = 5, 7
    for other in (copy.deepcopy(q), pickle.loads(pickle.dumps(q)), copy.copy(q)):
        assert other._at == (other.values.data_ptr(), other.scales.data_ptr())
        assert (other.format, other.shape, other.device) == (q.format, q.shape, q.device)
        assert np.all(other.values.array == 5) and np.all(other.scales.array == 7)
    assert copy.deepcopy(q)._at != q._at and copy.copy(q)._at == q._at


class Recorder:
    """A library whose calls succeed and are written down."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            if name == "ssgd_adamw_create":
                args[-1]._obj.value = 0x1234
            return args[0] * 128 if name == "ssgd_adamw_state_elements" else ssgd.OK
        return call


@pytest.fixture
def optimizer(fresh, monkeypatch):
    """(torch, the recorder, a function that makes an AdamW of three parameters and their copies)."""
    import contextlib
    torch = fresh

    class Parameter(torch.nn.Parameter):
        is_cuda = True
    recorder = Recorder()
    ssgd._load()
    monkeypatch.setattr(ssgd, "_lib", recorder)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(ssgd, "_call", lambda entry, device, *args: entry(*args))

    made = []

    def make(**more):
        params = [Parameter(torch.ones(n)) for n in (3, 0, 5)]
        made.append(ssgd.AdamW(params, **more))
        return params, made[-1]
    yield torch, recorder, make
    for opt in made:
        opt.close()          # (while the recorder is there: the handles are made up)


def test_an_optimizer_is_not_copied(optimizer):
    """A copy would free the first one's handle a second time."""
    torch, recorder, make = optimizer
    _, opt = make()
    for attempt in (copy.copy, copy.deepcopy, pickle.dumps):
        with pytest.raises(ssgd.SsgdError) as e:
            attempt(opt)
        assert e.value.status == ssgd.EINVAL and "adamw" in str(e.value)
    opt.close()
    opt.close()
    assert [name for name, _ in recorder.calls].count("ssgd_adamw_destroy") == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_assigned_moments_go_into_the_optimizers_own(optimizer, bits):
    """The handle keeps the addresses of the arrays that it was made with: moments that a program assigns are copied into them."""
    torch, _, make = optimizer
    _, opt = make(state_bits=bits)
    names = ["m", "v"] + (["m_scale", "v_scale"] if bits == 8 else [])
    places = {name: getattr(opt, name).data_ptr() for name in names}
    for k, name in enumerate(names):
        new = torch.full_like(getattr(opt, name), k + 1.0)
        setattr(opt, name, new)
        assert getattr(opt, name).data_ptr() == places[name] and torch.all(getattr(opt, name).float() == k + 1)
        for wrong in (new[:1], new.float().double(), None, 3.0):
            with pytest.raises(ssgd.SsgdError):
                setattr(opt, name, wrong)
    if bits == 32:
        opt.m_scale = opt.v_scale = None          # as a checkpoint of such an optimizer has them
        assert opt.m_scale is None and opt.v_scale is None
        with pytest.raises(ssgd.SsgdError):
            opt.m_scale = torch.zeros(3)
    opt.close()


def test_parameters_that_have_moved_are_refused(optimizer):
    """A parameter whose data was replaced (p.data = ..., a module that was converted) is no longer where the handle writes."""
    torch, recorder, make = optimizer
    copies = [torch.ones(3, dtype=torch.bfloat16), None, torch.ones(5, dtype=torch.bfloat16)]
    params, opt = make(copies=copies)
    grads = [torch.ones(n) for n in (3, 0, 5)]
    opt.step(grads, 0.1)
    steps = lambda: [name for name, _ in recorder.calls].count("ssgd_adamw_step")  # noqa: E731
    assert steps() == 1 and opt.t == 1
    for moved in (params[2], copies[0]):
        before = moved.data
        moved.data = before.clone()
        with pytest.raises(ssgd.SsgdError) as e:
            opt.step(grads, 0.1)
        assert e.value.status == ssgd.EINVAL and "moved" in str(e.value) and steps() == 1 and opt.t == 1
        moved.data = before
    opt.step(grads, 0.1)
    assert steps() == 2 and opt.t == 2
    opt.close()


def test_a_step_raises_the_version_counters(optimizer):
    torch, _, make = optimizer
    copies = [torch.ones(3, dtype=torch.bfloat16), None, None]
    params, opt = make(copies=copies)
    watched = [params[0], params[2], copies[0]]
    before = [t._version for t in watched]
    opt.step([torch.ones(n) for n in (3, 0, 5)], 0.1)
    assert all(t._version > b for t, b in zip(watched, before))
    opt.close()


def test_inputs_whose_gradient_would_be_lost_are_named(optimizer):
    """The operators record no graph: a tensor that requires a gradient is taken with a warning, and without one where no graph is wanted."""
    import warnings
    torch, _, _ = optimizer

    class Matrix(torch.nn.Parameter):
        is_cuda = True
    x, w = Matrix(torch.ones(4, 6)), Matrix(torch.ones(6))
    plain = Matrix(torch.ones(4, 6), requires_grad=False)
    for call in (lambda: ssgd._matrix(x, "an operator"), lambda: ssgd._weight(w, plain, "an operator"), lambda: ssgd._beside(x, plain, "an operator")):
        with pytest.warns(UserWarning, match="an operator.*no graph"):
            call()
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            with torch.no_grad():
                call()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        ssgd._matrix(plain, "an operator")
        ssgd._weight(w.detach(), plain, "an operator")
