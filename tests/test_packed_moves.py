"""A Packed is its tensors: calls take the addresses that these have at the call, whatever became of them since it was made; and it can be copied and pickled.

On the CPU: tensors that say they are on a GPU, and an entry point that writes down what it is given.  On the GPU: the same with results."""
import copy
import pickle

import pytest
import torch

from paper_1509_03371_amd import binding as B


class Claimed(torch.Tensor):
    """A CPU tensor that says it is on a GPU."""

    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.device.index

    def new_empty(self, *args, **kwargs):
        return super().new_empty(*args, **kwargs).as_subclass(Claimed)


def claimed(*shape, dtype=torch.uint8):
    return torch.zeros(shape, dtype=dtype).as_subclass(Claimed)


@pytest.fixture
def given(monkeypatch):
    """Addresses of codes and scales, as the entry points get them."""
    seen = []

    library = B.lib

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_workspace"):
                return getattr(library, name)

            def call(*args):
                for a in args:
                    if isinstance(getattr(a, "_obj", None), B.SkPacked):
                        seen.append((a._obj.codes, a._obj.scales))
                return 0
            return call

    monkeypatch.setattr(B, "lib", Lib())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    return seen


def calls(p, shape):
    """Every call that takes a Packed."""
    x = claimed(*shape, dtype=torch.float32)
    rstd, dw = claimed(shape[0], dtype=torch.float32), claimed(shape[1], shape[1], dtype=torch.float32)
    return [lambda: B.pack8(x, axis=1, out=p), lambda: B.unpack8(p, out=x), lambda: B.rms_norm(x, axis=1, y8=p, rstd=rstd), lambda: B.rms_norm(x, axis=1, sum8=p, rstd=rstd),
            lambda: B.rms_norm_backward(x, p, rstd, axis=1, parameters=False), lambda: B.weight_gradient8(x, p, bias=False, dw=dw)]


@pytest.mark.parametrize("how", ["other codes", "other scales", "both", "set_", "deepcopy", "pickle"])
def test_addresses_are_those_of_the_call(given, how):
    p = B.Packed(claimed(6, 70), claimed(6, 3), "i8", axis=1)
    keep = [p.codes, p.scales]                        # so that no address is taken again
    if how in ("other codes", "both"):
        p.codes = claimed(6, 70)
    if how in ("other scales", "both"):
        p.scales = claimed(6, 3)
    if how == "set_":
        p.codes.set_(torch.ones(6, 70, dtype=torch.uint8))
    if how == "deepcopy":
        p = copy.deepcopy(p)
    if how == "pickle":
        p = pickle.loads(pickle.dumps(p))
    for call in calls(p, (6, 70)):
        del given[:]
        call()
        assert given == [(p.codes.data_ptr(), p.scales.data_ptr())]
    assert len(keep) == 2


def test_what_does_not_fit_any_more_is_refused(given):
    def broken(change, error):
        p = B.Packed(claimed(6, 70), claimed(6, 3), "i8", axis=1)
        change(p)
        for call in calls(p, (6, 70)):
            with pytest.raises(error):
                call()
        assert not given

    broken(lambda p: setattr(p, "codes", torch.zeros(6, 70, dtype=torch.uint8)), TypeError)          # moved to the host
    broken(lambda p: setattr(p, "scales", torch.zeros(6, 3, dtype=torch.uint8)), TypeError)
    broken(lambda p: setattr(p, "scales", None), TypeError)
    broken(lambda p: setattr(p, "codes", claimed(6, 70, dtype=torch.int8)), TypeError)
    broken(lambda p: setattr(p, "scales", claimed(6, 2)), ValueError)
    broken(lambda p: setattr(p, "codes", claimed(5, 70)), ValueError)
    broken(lambda p: setattr(p, "code", "e5m2"), ValueError)
    broken(lambda p: p.codes.resize_(6, 69), ValueError)
    broken(lambda p: p.scales.resize_(0), ValueError)


def test_what_is_refused_from_the_start():
    for args, error in (((None, claimed(6, 3)), TypeError), ((claimed(6, 70), None), TypeError), ((torch.zeros(6, 70, dtype=torch.uint8), claimed(6, 3)), TypeError),
                        ((claimed(6, 70), claimed(6, 3), "e5m2"), ValueError), ((claimed(6, 70), claimed(6, 3), "i8", 2), ValueError),
                        ((claimed(6, 70), claimed(6, 3), "i8", -3), ValueError), ((claimed(6, 70), claimed(6, 2)), ValueError)):
        with pytest.raises(error):
            B.Packed(*args)
    assert B.Packed(claimed(6, 70), claimed(6, 3), "i8", -1).order == B.Packed(claimed(6, 70), claimed(6, 3), "i8", 1).order == (B.SK_ROWS, 6, 70, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(300, 90), (2, 40, 77)], ids=str)
def test_moved_to_the_host_and_back(shape):
    x, dz = torch.randn(shape, device="cuda"), torch.randn(shape[:1] + (11,) + shape[2:], device="cuda")
    p = B.pack8(x, "e4m3", axis=1)
    _, _, rstd = B.rms_norm(x, axis=1)

    def results(q):
        return [B.unpack8(q), *B.weight_gradient8(dz, q), *B.rms_norm_backward(x, q, rstd, axis=1)]

    want = [t.clone() for t in results(p)]
    q = pickle.loads(pickle.dumps(p))
    q.codes, q.scales = p.codes.cpu(), p.scales.cpu()
    with pytest.raises(TypeError):
        B.unpack8(q)
    for i in range(3):                                # where the tensors lay before holds others now
        q.codes, q.scales = q.codes.cpu(), q.scales.cpu()
        other = [torch.full_like(p.codes, 0x11) for _ in range(4)]
        q.codes, q.scales = q.codes.cuda(), q.scales.cuda()
        assert all(torch.equal(a, b) for a, b in zip(results(q), want)), i
        assert all((t == 0x11).all() for t in other)
    r = copy.deepcopy(p)
    B.pack8(2 * x, axis=1, out=r)
    assert all(torch.equal(a, b) for a, b in zip(results(p), want)), "a copy shares nothing"
    assert torch.equal(B.unpack8(r).float(), 2 * B.unpack8(p).float())
