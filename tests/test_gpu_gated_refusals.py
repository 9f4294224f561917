"""What the binding of the RMS norm and the gated layer says of tensors that it cannot pass on: the argument and the reason (those of the entry
points themselves: test_operator_refusals.py)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2105_13336_amd as P  # noqa: E402

INVAL = P.binding.TENSILE_E_INVAL


@pytest.fixture(scope="module")
def ops():
    h = P.tensile_ops_create()
    yield h
    h.close()


def refused(call, begins):
    with pytest.raises(P.TensileError) as e:
        call()
    assert e.value.code == INVAL and begins in str(e.value) and f" {begins}" in f" {e.value}", str(e.value)


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


MATRIX = "need a CUDA tensor on the handle's device (0), of float32, bfloat16 or float16, with at least one dimension"
VECTOR = "need a contiguous CUDA tensor on the handle's device (0), of torch.{} with {} elements"


def test_norm(ops):
    x, y, g, rstd, c = zeros(4, 64), zeros(4, 64), zeros(64, dtype=torch.float32), zeros(4, dtype=torch.float32), P.Checkpoint.empty(4, 64)
    norm, back = P.tensile_rms_norm, P.tensile_rms_norm_backward
    refused(lambda: norm(ops, x.cpu(), g, y), "x: " + MATRIX)
    refused(lambda: norm(ops, x, g, y.int()), "y: " + MATRIX)
    refused(lambda: norm(ops, x, g, y, residual=x.cpu()), "residual: " + MATRIX)
    refused(lambda: norm(ops, x, g, y, total=x.double()), "total: " + MATRIX)
    refused(lambda: norm(ops, x, g, zeros(64, 4).t()), "y: the columns of a row have to be contiguous")
    refused(lambda: norm(ops, x, g[:63], y), "gamma: " + VECTOR.format("float32", 64))
    refused(lambda: norm(ops, x, g.cpu(), y), "gamma: " + VECTOR.format("float32", 64))
    refused(lambda: norm(ops, x, zeros(128, dtype=torch.float32)[::2], y), "gamma: " + VECTOR.format("float32", 64))
    refused(lambda: norm(ops, x, g, y, rstd=rstd[:3]), "rstd: " + VECTOR.format("float32", 4))
    refused(lambda: norm(ops, x, g, y, rstd=rstd.double()), "rstd: " + VECTOR.format("float32", 4))
    refused(lambda: norm(ops, x, g, None), "rms_norm: y is NULL")
    refused(lambda: norm(ops, x, g, x[:, :1].expand(4, 64)), "y: the columns of a row have to be contiguous")
    refused(lambda: back(ops, x, c, rstd[:2], g, y), "rstd: " + VECTOR.format("float32", 4))
    refused(lambda: back(ops, x, c, rstd, g, y, dgamma=g[:60]), "dgamma: " + VECTOR.format("float32", 64))
    refused(lambda: back(ops, x, c, rstd, g, y, dgamma=zeros(64)), "dgamma: " + VECTOR.format("float32", 64))
    refused(lambda: back(ops, x, c, rstd, g, y, dresidual=x.cpu()), "dresidual: " + MATRIX)
    refused(lambda: back(ops, x, c, rstd, g, None), "rms_norm_backward: dx is NULL")


def test_gated(ops):
    x, w, h, c, d = zeros(4, 64), zeros(32, 64), zeros(4, 32), P.Checkpoint.empty(4, 32), P.Checkpoint.empty(4, 32)
    gated, back = P.tensile_gated_linear, P.tensile_gated_linear_backward
    refused(lambda: gated(ops, x.cpu(), w, w, h), "x: " + MATRIX)
    refused(lambda: gated(ops, x, w.cpu(), w, h), "w_gate: " + MATRIX)
    refused(lambda: gated(ops, x, w, w.long(), h), "w_up: " + MATRIX)
    refused(lambda: gated(ops, x, w, w, h.cpu()), "h: " + MATRIX)
    refused(lambda: gated(ops, x, w, w.t().contiguous().t(), h), "w_up: the columns of a row have to be contiguous")
    refused(lambda: gated(ops, x, w, w, h, b_gate=zeros(31), b_up=zeros(32)), "b_gate: " + VECTOR.format("bfloat16", 32))
    refused(lambda: gated(ops, x, w, w, h, b_gate=zeros(32), b_up=zeros(33)), "b_up: " + VECTOR.format("bfloat16", 32))
    refused(lambda: gated(ops, x, w, w, h, b_gate=zeros(32), b_up=zeros(32, dtype=torch.float32)), "b_up: " + VECTOR.format("bfloat16", 32))
    refused(lambda: gated(ops, x, w, w, h, act="relu"), "act: 'relu' is not one of silu, gelu, gelu_tanh")
    refused(lambda: gated(ops, x, w, w, x[:, 8:40]), "gated_linear: h overlaps x")
    refused(lambda: back(ops, h.cpu(), c, d, h, zeros(4, 32)), "dh: " + MATRIX)
    refused(lambda: back(ops, h, c, d, zeros(4, 32).cpu(), h), "dgate: " + MATRIX)
    refused(lambda: back(ops, h, c, d, h, h.cpu()), "dup: " + MATRIX)
    refused(lambda: back(ops, h, c, d, h, zeros(4, 32), w_gate=w, w_up=w, dx=x.cpu()), "dx: " + MATRIX)
    refused(lambda: back(ops, h, c, d, h, zeros(4, 32), act="tanh"), "act: 'tanh' is not one of silu, gelu, gelu_tanh")
    both = zeros(4, 64)
    refused(lambda: back(ops, both.view(8, 32)[:4], c, d, both[:, :32], zeros(4, 32)), "gated_linear_backward: dgate overlaps dh")
