"""What the torch side of the triangle update refuses before the library sees an address: tensors of another type,
shape, layout or device than the kernels take for granted.  The checks come first, so they run without a GPU."""
import pytest
import torch

from paper_2603_14806_amd import trimul as T

N = 6


def layer(dtype="bf16", out_dtype="f32"):
    """A layer without a handle: whatever gets past the checks fails with another error."""
    t = T.TriMul.__new__(T.TriMul)
    t.dtype, t.out_dtype, t.device, t.h, t._ws = dtype, out_dtype, torch.device("cpu"), None, None
    t._on = torch.device("cuda", 0)
    return t


def calls(t):
    dout = torch.zeros(N, N, 128, dtype=torch.bfloat16)
    return {"outgoing": t.outgoing, "incoming": t.incoming, "call": lambda z, m=None: t(z, m, "incoming"), "residual": t.residual,
            "residual_backward": lambda z, m=None: t.residual_backward(z, dout, m)}


Z = torch.zeros(N, N, 128, dtype=torch.bfloat16)
BAD = {"float32 on a bf16 layer": (Z.float(), None, "type"),
       "rows of a larger tensor": (torch.zeros(N, N + 3, 128, dtype=torch.bfloat16)[:, :N], None, "contiguous"),
       "rectangle": (torch.zeros(N, N + 1, 128, dtype=torch.bfloat16), None, "contiguous"),
       "too few channels": (torch.zeros(N, N, 64, dtype=torch.bfloat16), None, "contiguous"),
       "transposed": (Z.transpose(0, 1), None, "contiguous"),
       "short mask": (Z, torch.ones(N - 1, dtype=torch.uint8), "mask"),
       "float mask": (Z, torch.ones(N), "mask"),
       "strided mask": (Z, torch.ones(2 * N, dtype=torch.uint8)[::2], "mask"),
       "host memory": (Z, None, "GPU")}


@pytest.mark.parametrize("name", ["outgoing", "incoming", "call", "residual", "residual_backward"])
@pytest.mark.parametrize("what", BAD)
def test_refused(name, what):
    z, mask, word = BAD[what]
    with pytest.raises(ValueError, match=word):
        calls(layer())[name](z, mask)


def test_bf16_on_a_float32_layer():
    """The kernels would read twice the memory that is there."""
    for name in ("outgoing", "incoming", "residual"):
        with pytest.raises(ValueError, match="type"):
            calls(layer("f32"))[name](Z)


def test_outputs_refused():
    for name in ("outgoing", "incoming"):
        for out, word in ((torch.zeros(N, N, 128, dtype=torch.bfloat16), "out must be of the layer's type"),
                          (torch.zeros(N, N + 1, 128)[:, :N], "out must be a contiguous")):
            with pytest.raises(ValueError, match=word):
                getattr(layer(), name)(Z, None, out)
