"""What the binding asks of the tensors of calls without a state before it calls the library: stand-ins, no GPU, addresses that are never read."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2605_26444_amd import binding as B

P = 1 << 20


class Stub:
    """stands for a device tensor"""
    is_cuda = True

    def __init__(self, device=0, shape=(4, 32), dtype=torch.float32, stride=None):
        self.device_index, self.shape, self.dtype, self.strides = device, shape, dtype, stride or (shape[1] if len(shape) > 1 else 1, 1)[2 - len(shape):]

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self):
        return self.strides


@pytest.fixture(autouse=True)
def on_device_0(monkeypatch):
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_26444_amd import build
        build.build()
    B.lib()
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda stream: 0)


def rows(**k):
    """rows of logits of device 0; k: tensors in place of its own"""
    a = {**dict(z=Stub(), t=Stub(shape=(4,), dtype=torch.int32), ids=None, n=None), **k}
    return B.logit_rows(a["z"], a["t"], ids=a["ids"], n=a["n"])


# calls with sizes that the library refuses, so that nothing is launched whatever the tensors are: NanoSpecError says that the binding let them pass
CALLS = {
    "quantize": (("X", "Q", "scale"), lambda a: B.nanospec_quantize_rows(a["X"], 0, 16, a["Q"], a["scale"])),
    "head": (("W", "S", "H", "out", "ws"), lambda a: B.nanospec_dense_head_i8(a["W"], a["S"], a["H"], 0, 16, 1, a["out"], a["ws"], 1 << 30)),
    "logprob": (("lp", "ws"), lambda a: B.nanospec_token_logprob(rows(), a["lp"], a["ws"], 0)),
    "policy": (("old", "ref", "adv", "w", "loss", "row", "lp", "grad", "ws"),
               lambda a: B.nanospec_policy_loss(rows(), a["old"], a["ref"], a["adv"], a["w"], -1.0, 0.2, 0.1, a["loss"], a["row"], a["lp"], a["grad"], a["ws"], 0)),
    "preference": (("ref", "w", "loss", "margin", "lp", "grad", "ws"),
                   lambda a: B.nanospec_preference_loss(rows(), [0, 1, 2], a["ref"], a["w"], 0.1, -1.0, a["loss"], a["margin"], a["lp"], a["grad"], a["ws"], 0)),
}


@pytest.mark.parametrize("call,name", [(c, n) for c, (names, _) in CALLS.items() for n in names])
def test_every_tensor_is_the_current_devices(call, name):
    names, run = CALLS[call]
    with pytest.raises(B.NanoSpecError):
        run({n: Stub() for n in names})
    with pytest.raises(ValueError, match="device 3"):
        run({n: Stub(3 if n == name else 0) for n in names})
    with pytest.raises(ValueError, match="device -1"):      # host memory
        run({n: Stub(-1 if n == name else 0) for n in names})


@pytest.mark.parametrize("name", ["t", "ids", "n"])
def test_rows_of_logits_are_one_devices(name):
    rows(), rows(ids=Stub(shape=(4,)), n=Stub(shape=(4,))), rows(ids=P, n=P)
    with pytest.raises(ValueError, match="device 3"):
        rows(**{"ids": P, "n": P, name: Stub(3, shape=(4,), dtype=torch.int32)})


@pytest.mark.parametrize("call", [lambda r: B.nanospec_token_logprob(r, P, P, 0), lambda r: B.nanospec_policy_loss(r, P, P, P, None, -1.0, 0.2, 0.1, P, None, None, None, P, 0),
                                  lambda r: B.nanospec_preference_loss(r, [0, 1, 2], None, None, 0.1, -1.0, P, None, None, None, P, 0)])
def test_rows_of_logits_of_another_device(call):
    there = rows(z=Stub(3), t=Stub(3, shape=(4,), dtype=torch.int32))
    with pytest.raises(ValueError, match="device 3"):
        call(there)
    with pytest.raises(B.NanoSpecError):
        call(rows())


@pytest.mark.parametrize("shape,stride", [((4, 32), None), ((4, 32), (64, 1)), ((1, 32), (64, 1))])
def test_no_more_columns_than_the_logits_have(shape, stride):
    """a wider row stride, or a single row, is no room for more columns: the last row's would lie behind the tensor"""
    z, t = Stub(shape=shape, stride=stride), Stub(shape=(4,), dtype=torch.int32)
    assert B.logit_rows(z, t).V == 32 and B.logit_rows(z, t, V=31).V == 31
    for V in (33, 64):
        with pytest.raises(ValueError, match="columns"):
            B.logit_rows(z, t, V=V)
