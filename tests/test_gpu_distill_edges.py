"""Top logits and the distillation loss where their rules change: workspaces of exactly the bytes that are asked for, masked
pieces of rows far from zero, a loss of labels alone."""
import numpy as np
import pytest
import torch

from tests.test_gpu_distill import matrix, top_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_1912_12675_amd import psw
    psw.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return psw


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("n,c,k,type_", [(2, 262144, 128, "f32"), (2, 524288, 64, "f32"), (2, 524288, 128, "bf16"),
                                         (1, 1 << 20, 32, "f32"), (3, 1 << 20, 64, "bf16"), (2, 131072, 128, "f32")])
def test_top_logits_workspace(P, n, c, k, type_, pad):
    """Around 8192 keys to merge, where 16 bytes more or less of a row choose other pieces: a workspace of the bytes that
    are asked for is enough, and what lies behind it stays."""
    print(f"top_logits workspace {n}x{c} k {k} {type_} pad {pad}", flush=True)
    rng = np.random.default_rng(c + k)
    z, _ = matrix(rng.standard_normal((n, c)) * 3, type_, pad)
    need, guard = P.psw_top_logits_ws_bytes(n, c, k), 1 << 20
    buf = torch.full((need + guard,), 171, dtype=torch.uint8, device="cuda")
    val, idx, lse = torch.zeros(n, k, device="cuda"), torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    P.psw_top_logits(z, val, idx, lse=lse, ws=buf[:need])
    torch.cuda.synchronize()
    assert bool((buf[need:] == 171).all())
    v, order, want = top_ref(z.double().cpu().numpy(), k, 1.0)
    np.testing.assert_array_equal(idx.cpu().numpy(), order)
    np.testing.assert_array_equal(val.double().cpu().numpy(), v)
    # as in check_top: 300 half steps of the terms' sum, and one rounding
    assert (np.abs(lse.double().cpu().numpy() - want) <= 300 * 2.0**-24 + 2.0**-24 * np.abs(want)).all()
