"""Calls of the 8-bit products and the norms whose arrays lie on different devices, or hold fewer elements than the call writes, are refused ahead
of the library.  No GPU is needed: stand-ins take the arrays' place, and a call that passes the checks is refused by the library for its
missing context."""
import pytest
import torch

from paper_2510_05528_b200 import binding as Bd
from paper_2510_05528_b200 import build as armor_build

BF16, F32, I8, U8 = torch.bfloat16, torch.float32, torch.int8, torch.uint8
N, D = 6, 64


class Array:
    """What the binding asks of a tensor, of a contiguous one on a GPU."""
    is_cuda = True

    def __init__(self, *shape, dtype=BF16, device=0):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", device)
        self._stride = torch.empty(shape, device="meta").stride()

    def get_device(self):
        return self.device.index

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def size(self, i):
        return self.shape[i]

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 0x10000

    def unsqueeze(self, i):
        return Array(1, *self.shape, dtype=self.dtype, device=self.device.index)

    def moved(self):
        return Array(*self.shape, dtype=self.dtype, device=1)


def rows(dtype=BF16):
    return Array(N, D, dtype=dtype)


def vector(n=D):
    return Array(n, dtype=F32)


CALLS = {
    "quantize_rows": (lambda **t: Bd.armor_quantize_rows(None, t["x"], t["q"], t["scale"]), {"x": rows(), "q": rows(I8), "scale": vector(N)}),
    "linear_i8": (lambda **t: Bd.armor_linear_i8(None, t["x"], None, t["wq"], t["w_scale"], t["bias"], t["y"]),
                  {"x": rows(), "wq": Array(32, D, dtype=I8), "w_scale": vector(32), "bias": vector(32), "y": Array(N, 32)}),
    "linear_i8_given": (lambda **t: Bd.armor_linear_i8(None, t["x"], t["x_scale"], t["wq"], t["w_scale"], None, t["y"]),
                        {"x": rows(I8), "x_scale": vector(N), "wq": Array(32, D, dtype=I8), "w_scale": vector(32), "y": Array(N, 32)}),
    "apply_layer_i8": (lambda **t: Bd.armor_apply_layer_i8(None, t["packed"], t["x"], t["y"]), {"packed": Array(999, dtype=U8), "x": rows(), "y": rows()}),
    "block_norm": (lambda **t: Bd.armor_block_norm(None, t["x"], t["y"], t["h"], t["n"], t["q"], t["q_scale"], gate=t["gate"], w_post=t["w_post"], w_pre=t["w_pre"]),
                   {**{k: rows() for k in ("x", "y", "h", "n")}, "q": rows(I8), "q_scale": vector(N), **{k: vector() for k in ("gate", "w_post", "w_pre")}}),
    "block_norm_backward": (lambda **t: Bd.armor_block_norm_backward(None, *[t[k] for k in ("h", "y", "dh", "dn", "dx", "dy", "dw_post", "dw_pre", "dgate")], gate=t["gate"],
                                                                     w_post=t["w_post"], w_pre=t["w_pre"]),
                            {**{k: rows() for k in ("h", "y", "dh", "dn", "dx", "dy")}, **{k: vector() for k in ("dw_post", "dw_pre", "dgate", "gate", "w_post", "w_pre")}}),
}


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    armor_build.build()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(Bd, "_stream", lambda: 0)


@pytest.mark.parametrize("name", CALLS)
def test_one_device(name, monkeypatch):
    call, arrays = CALLS[name]
    with pytest.raises(Bd.ArmorError):                     # (the library: no context)
        call(**arrays)
    for moved in arrays:
        with pytest.raises(ValueError, match="cuda:"):
            call(**{**arrays, moved: arrays[moved].moved()})
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        call(**arrays)


@pytest.mark.parametrize("name", CALLS)
def test_arrays_of_too_few_elements(name):
    """An output or a vector without columns, or a row short; the first array says how many there are."""
    call, arrays = CALLS[name]
    for k, t in list(arrays.items())[1:]:
        if k == "packed":
            continue
        less = [Array(*t.shape[:-1], 0, dtype=t.dtype)] if t.dim() == 1 else [Array(t.shape[0] - 1, *t.shape[1:], dtype=t.dtype)]
        if t.dim() == 1:
            less.append(Array(*t.shape, 0, dtype=t.dtype))
        for v in less:
            if k in ("x", "wq") and name in ("apply_layer_i8", "linear_i8", "linear_i8_given"):
                continue                                   # (others would have to follow)
            with pytest.raises(ValueError):
                call(**{**arrays, k: v})


def test_what_another_call_packed():
    """A core, a layer and a layer in 8 bits are bytes alike: each forward refuses what is too small for it, and the 8-bit one whatever is
    not its own."""
    ctx = object.__new__(Bd.ArmorContext)
    ctx.cfg, ctx.d_out, ctx.d_in, ctx._index, ctx._sizes, ctx.device = Bd.make_config(512, 768, 128), 512, 768, 0, {}, torch.device("meta")
    core, layer, layer8 = (torch.empty(f(ctx.cfg), dtype=U8) for f in (Bd.armor_packed_core_bytes, Bd.armor_packed_layer_bytes, Bd.armor_packed_layer_i8_bytes))
    x = Array(3, 768)
    for call, mine, wrong in ((lambda p: ctx.apply_packed(None, p, x), "pack_core", [core[:-1], core.view(torch.int8)]),
                              (lambda p: ctx.apply_layer(p, x), "pack_layer", [core, layer8, layer[1:], layer.float()]),
                              (lambda p: ctx.apply_layer_i8(p, x), "pack_layer_i8", [core, layer, layer8[1:], layer8.view(torch.int8)])):
        for p in wrong:
            with pytest.raises(ValueError, match=f"what {mine} made"):
                call(p)
    with pytest.raises(ValueError, match="on meta"):       # (of the right size, and in host memory)
        ctx.apply_layer_i8(layer8, x)
