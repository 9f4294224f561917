"""The operators on 8-bit checkpoints at the edges of what their entry points allow, against plain statements or the ordinary form of the
same call."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2105_13336_amd as P  # noqa: E402
from test_gpu_ops import check_grad, filled, host, near, say, up  # noqa: E402

TYPES = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def ops():
    h = P.tensile_ops_create()
    yield h
    h.close()


# ------------------------------------------------------------------ weight gradient

def spread(c, ld_q=None, ld_s=None):
    """The same checkpoint with its rows further apart (what lies between them is never written)."""
    def far(t, ld):
        if ld is None:
            return t
        v = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (ld, 1))
        v.copy_(t)
        return v
    return P.Checkpoint(far(c.q, ld_q), far(c.scale, ld_s))


# 31 rows of a step: from 2^32 / 31 = 138,547,333 bytes between rows a row's offset needs more than 32 bits
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,far", [(3, dict(ld_s=2 ** 31)), (3, dict(ld_q=2 ** 31)), (40, dict(ld_s=2 ** 27 + 2 ** 23)), (40, dict(ld_q=2 ** 26 - 1, ld_s=2 ** 26)),
                                   (170, dict(ld_s=2 ** 27 + 2 ** 23)), (200, dict(ld_q=2 ** 20, ld_s=2 ** 26 - 1))])
def test_linear_grad_of_far_apart_rows(ops, dtype, M, far):
    """Pitches of the bytes and of the scales on both sides of what 32-bit offsets reach."""
    say(f"linear grad {dtype} {M} rows {far}")
    rng = np.random.default_rng(M)
    c, x = filled(rng.standard_normal((M, 72)) * np.exp2(rng.integers(-9, 9, (M, 1))))
    dy = up(rng.standard_normal((M, 72)), dtype)
    dw = torch.empty(72, 72, device="cuda")
    wide = spread(c, **far)
    P.tensile_linear_grad(ops, dy, wide, dw)
    want, size = host(dy).T @ x, np.abs(host(dy)).T @ np.abs(x)
    near(dw, want, (M / 16 + 90) * 2.0 ** -24 * size, "dw")
    del wide
    torch.cuda.empty_cache()
