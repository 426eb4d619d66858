"""What the binding of the training operators refuses before it calls the library, without a GPU: tensors of another device than the
context's, which a kernel may not read.  The tensors here say that they are on a device and hold nothing."""
import pytest
import torch

from paper_2301_06051_b200 import api


class Tensor:
    """A contiguous tensor on device `at` as far as the binding asks."""

    def __init__(self, shape, dtype, at):
        self._meta, self.at = torch.empty(shape, dtype=dtype, device="meta"), at
        self.shape, self.dtype, self.is_cuda = self._meta.shape, dtype, at >= 0

    def get_device(self):
        return self.at

    def data_ptr(self):
        return 4096

    def __getattr__(self, name):  # stride, numel, dim, is_contiguous
        return getattr(self._meta, name)


class Library:
    """Counts calls, launches nothing."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return api.OK
        return call


def _context(at):
    ctx = object.__new__(api.Context)
    ctx.lib, ctx._h, ctx.device, ctx._index, ctx._raw_stream, ctx._current = Library(), None, torch.device("cuda", at), at, 0, lambda i: 0
    return ctx


def _attention(at, odd=None, other=1):
    """Arguments of both attention calls, `odd` of them on device `other`."""
    n, heads, dim, where = 40, 2, 16, lambda name: other if name == odd else at
    t = {m: Tensor((n, heads, dim), torch.float32, where(m)) for m in ("q", "k", "v", "do", "out", "dq", "dk", "dv")}
    for m, shape in (("start", (5,)), ("order", (n,)), ("coords", (n, 4)), ("num", (1,))):
        t[m] = Tensor(shape, torch.int32, where(m))
    t["table"], t["dbias"] = Tensor((heads, 9), torch.float32, where("table")), Tensor((heads, 9), torch.float32, where("dbias"))
    seg = api.Segments(t["start"], 12, t["order"], t["coords"], t["num"])
    return t, seg, api.BucketBias(t["table"], (2, 2, 1), [0] * 7)


@pytest.mark.parametrize("at", [0, 1])
def test_tensors_on_the_contexts_device_go_through(at):
    ctx = _context(at)
    t, seg, rel = _attention(at)
    ctx.segment_attention(t["q"], t["k"], t["v"], seg, bias=rel, out=t["out"])
    ctx.segment_attention_backward(t["q"], t["k"], t["v"], t["do"], seg, bias=rel, out=(t["dq"], t["dk"], t["dv"]), dbias=t["dbias"])
    x, g = Tensor((40, 32), torch.float32, at), Tensor((32,), torch.float32, at)
    ctx.layer_norm(x, g, g, residual=x, out=x)
    ctx.layer_norm_backward(x, x, g, residual=x, out=x, dg=g, db=g)
    assert ctx.lib.calls == 4


@pytest.mark.parametrize("at,other", [(0, 1), (1, 0), (0, -1)])
@pytest.mark.parametrize("odd", ["q", "k", "v", "out", "start", "order", "coords", "num", "table"])
def test_attention_refuses_tensors_of_another_device(at, other, odd):
    ctx = _context(at)
    t, seg, rel = _attention(at, odd, other)
    with pytest.raises(ValueError, match="device"):
        ctx.segment_attention(t["q"], t["k"], t["v"], seg, bias=rel, out=t["out"])
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("at,other", [(0, 1), (1, 0), (0, -1)])
@pytest.mark.parametrize("odd", ["q", "k", "v", "do", "dq", "dk", "dv", "dbias", "start", "order", "coords", "num", "table"])
def test_its_backward_pass_refuses_tensors_of_another_device(at, other, odd):
    ctx = _context(at)
    t, seg, rel = _attention(at, odd, other)
    with pytest.raises(ValueError, match="device"):
        ctx.segment_attention_backward(t["q"], t["k"], t["v"], t["do"], seg, bias=rel, out=(t["dq"], t["dk"], t["dv"]), dbias=t["dbias"])
    assert ctx.lib.calls == 0


@pytest.mark.parametrize("at,other", [(0, 1), (1, 0), (0, -1)])
@pytest.mark.parametrize("odd", ["x", "r", "dy", "g", "b", "out", "dg", "db"])
def test_layer_norm_refuses_tensors_of_another_device(at, other, odd):
    ctx = _context(at)
    t = {m: Tensor((40, 32) if m in ("x", "r", "dy", "out") else (32,), torch.float32, other if m == odd else at)
         for m in ("x", "r", "dy", "g", "b", "out", "dg", "db")}
    if odd not in ("dy", "dg", "db"):
        with pytest.raises(ValueError, match="device"):
            ctx.layer_norm(t["x"], t["g"], t["b"], residual=t["r"], out=t["out"])
    if odd != "b":
        with pytest.raises(ValueError, match="device"):
            ctx.layer_norm_backward(t["x"], t["dy"], t["g"], residual=t["r"], out=t["out"], dg=t["dg"], db=t["db"])
    assert ctx.lib.calls == 0
