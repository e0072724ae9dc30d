"""The binding refuses tensors of the documented number of elements in another order, before any launch.  The tensors are
stand-ins that say they are on a device: nothing reads them."""
import numpy as np
import pytest
import torch

from paper_2609_34318_amd import hydra

BF16, F32 = torch.bfloat16, torch.float32


class Stand:
    is_cuda = True

    def __init__(self, *shape, dtype=BF16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def is_contiguous(self):
        return True

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.dtype.itemsize

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 20


@pytest.fixture(autouse=True)
def _device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    def unreached():
        raise AssertionError("the library was called")
    monkeypatch.setattr(hydra, "_stream", lambda s: unreached())


T, H, D = 6, 4, 64
NORM = {"x": (2, T, H // 2, D), "y": (T, H, D), "weight": (H, D), "bias": (H, D), "gate": (T, H, D), "d_y": (T, H, D),
        "d_x": (2, T, H // 2, D), "d_gate": (T, H, D), "d_weight": (H, D), "d_bias": (H, D)}


def norm_tensors(**other):
    f32 = ("weight", "bias", "d_weight", "d_bias")
    return {n: Stand(*other.get(n, s), dtype=F32 if n in f32 else BF16) for n, s in NORM.items()}


def unpack(t):
    hydra.unpack_heads_normed(t["x"], t["y"], t["weight"], t["bias"], t["gate"])


def pack(t):
    hydra.pack_heads_normed_bwd(t["x"], t["d_y"], t["d_x"], t["weight"], t["bias"], t["gate"], t["d_gate"], t["d_weight"],
                                t["d_bias"], Stand(1 << 20, dtype=torch.uint8))


@pytest.mark.parametrize("name,shape", [
    ("gate", (H, T, D)), ("y", (H, T, D)), ("weight", (D, H)), ("bias", (D, H)), ("y", (T, D, H)), ("y", (T, H * D)),
    ("d_y", (H, T, D)), ("d_gate", (H, T, D)), ("d_x", (2, H // 2, T, D)), ("d_x", (T, H, D)), ("d_weight", (D, H)),
    ("d_bias", (D, H))])
def test_norm(name, shape):
    t = norm_tensors(**{name: shape})
    for call, takes in ((unpack, name not in ("d_y", "d_x", "d_gate", "d_weight", "d_bias")), (pack, name != "y")):
        if takes:
            with pytest.raises(ValueError, match=f"{name}: shape"):
                call(t)


def test_norm_takes_what_is_documented():
    """The documented shapes, and weight and bias as one row of all heads' channels, reach the library."""
    for flat in ({}, {n: (H * D,) for n in ("weight", "bias", "d_weight", "d_bias")}):
        for call in (unpack, pack):
            with pytest.raises(AssertionError, match="called"):
                call(norm_tensors(**flat))


STEP = {"q": (T, H, D), "k": (T, 2, D), "v": (T, 2, 128), "o": (T, H, 128), "state": (9, H, D, 128), "state_out": (9, H, D, 128)}


def step(**other):
    t = {n: Stand(*other.get(n, s), dtype=F32 if "state" in n else BF16) for n, s in STEP.items()}
    hydra.linear_step(t["q"], t["k"], t["v"], Stand(H, dtype=F32), t["state"], t["o"], Stand(T, dtype=torch.int32), t["state_out"])


@pytest.mark.parametrize("name,shape", [("k", (2, T, D)), ("k", (T, D, 2)), ("v", (T * 2, 1, 128)), ("o", (H, T, 128)), ("o", (T, 128, H)),
                                        ("o", (T, H * 128)), ("state", (H, 9, D, 128)), ("state_out", (9, D, H, 128))])
def test_step(name, shape):
    with pytest.raises(ValueError, match="shape"):
        step(**{name: shape})
    with pytest.raises(AssertionError, match="called"):
        step()


LINEAR = {"q": (T, H, D), "k": (T, 2, D), "v": (T, 2, 128), "o": (T, H, 128), "state_in": (2, H, D, 128), "state_out": (2, H, D, 128),
          "d_state_out": (2, H, D, 128), "d_state_in": (2, H, D, 128)}


@pytest.mark.parametrize("name,shape", [("state_in", (H, 2, D, 128)), ("state_in", (2, H, 128, D)), ("state_out", (2, D, H, 128)),
                                        ("d_state_out", (H, 2, D, 128)), ("d_state_in", (2, H, 128, D)), (None, None)])
def test_linear_states(name, shape):
    t = {n: Stand(*(shape if n == name else s), dtype=F32 if "state" in n else BF16) for n, s in LINEAR.items()}
    p = hydra.Linear([0, 2, T], H, D, 128, n_kv_heads=2)
    ws, decay = Stand(1 << 20, dtype=torch.uint8), Stand(H, dtype=F32)

    def fwd():
        hydra.linear_fwd(p, t["q"], t["k"], t["v"], decay, t["o"], ws, t["state_in"], t["state_out"])

    def bwd():
        hydra.linear_bwd(p, t["q"], t["k"], t["v"], decay, t["o"], t["q"], t["k"], t["v"], ws, t["state_in"], t["d_state_out"],
                         t["d_state_in"])
    for call, takes in ((fwd, ("state_in", "state_out")), (bwd, ("state_in", "d_state_out", "d_state_in"))):
        with pytest.raises(ValueError if name in takes else AssertionError, match=f"{name}: shape" if name in takes else "called"):
            call()
