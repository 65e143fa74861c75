"""What the torch side of the triangle update refuses before the library sees an address: tensors of another type,
shape, layout or device than the kernels take for granted.  The checks come first, so they run without a GPU."""
import pytest
import torch

from paper_2603_14806_amd import trimul as T

N = 6


def layer(dtype="bf16", out_dtype="f32"):
    """A layer without a handle: whatever gets past the checks fails with another error."""
    t = T.TriMul.__new__(T.TriMul)
    t.dtype, t.out_dtype, t.device, t.h, t._ws = dtype, out_dtype, torch.device("cpu"), None, {}
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


def test_workspaces_by_stream_and_capture(monkeypatch):
    """Calls on two streams may run at once and a graph keeps the memory it was captured with, so neither shares a
    workspace; calls on one stream, outside of a capture, do (what a call leaves there can be read)."""
    at, used = [(1, False)], []
    monkeypatch.setattr(T, "_place", lambda device: at[0], raising=False)
    monkeypatch.setattr(T, "tri_mul_workspace_size", lambda h, n: 4096 * n)
    monkeypatch.setattr(T, "_stream", lambda s: at[0][0])

    class Here:
        def __init__(self, *a): pass
        def __enter__(self): return at[0][0]
        def __exit__(self, *a): pass

    def update(h, z, mask, n, out, ws, need, stream):
        assert ws.numel() >= need == 4096 * n
        used.append(ws)
    monkeypatch.setattr(T, "on_stream", Here)
    monkeypatch.setattr(T, "tri_mul_outgoing", update)
    t = layer()
    t._on, t._ws = torch.device("cpu"), {}

    def call(place, n):
        at[0] = place
        t.outgoing(torch.zeros(n, n, 128, dtype=torch.bfloat16))
        assert t.workspace(n)[0].data_ptr() == used[-1].data_ptr()
        return used[-1].data_ptr()
    a, b = call((1, False), 8), call((2, False), 8)
    assert a != b and call((1, False), 8) == a and call((2, False), 4) == b
    graphs = [call((1, True), 8), call((1, True), 8), call((2, True), 4)]
    assert len({a, b, *graphs}) == 5                   # (all are held here)
    assert call((1, False), 8) == a
    assert call((1, False), 9) not in (a, b, *graphs)


def test_gradients_on_another_device_are_refused():
    """The kernels run on the layer's GPU, on addresses of whichever device dout is on."""
    t = layer()
    t._on = torch.device("meta")
    z, dout = Z.to("meta"), torch.zeros(N, N, 128)
    for f in (t.backward, t.residual_backward):
        with pytest.raises(ValueError, match="dout must live on the GPU of the layer"):
            f(z, dout)
