"""Top logits and the distillation loss where their rules change: workspaces of exactly the bytes that are asked for, masked
pieces of rows far from zero, a loss of labels alone."""
import numpy as np
import pytest
import torch

from tests.test_gpu_distill import TYPES, check_distill, check_top, distill_ref, matrix, run, teacher, top_ref

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


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,k,pad,tau,at,spread,masked", [
    (2, 70000, 5, 0, 0.046875, -8.6, 0.0, 464),      # a short last piece that a mask covers
    (3, 262144, 40, 0, 1.0, -1000.0, 3.0, 100000),
    (130, 140000, 3, 1, 2.0**-7, -5.0, 1.0, 70000),
    (2, 131072, 128, 1, 1.0, -300.0, 3.0, 0),    # rows that begin inside 16 bytes have a piece more, the others' is empty
    (1, 1 << 20, 256, 0, 2.0**-16, -1.0, 0.5, 1 << 19)])
def test_masked_pieces_far_from_zero(P, n, c, k, pad, tau, at, spread, masked, type_):
    """Pieces of a row that hold nothing, and a largest logit below -89 T: the exponential of its distance from 0 has no
    number, and is not to be multiplied by the empty piece's sum."""
    print(f"masked pieces {n}x{c} k {k} {type_} pad {pad} T {tau} at {at}", flush=True)
    rng = np.random.default_rng(c)
    z = at + rng.standard_normal((n, c)) * spread
    z[:, c - masked:] = -np.inf
    x, _ = matrix(z, type_, pad)
    check_top(P, x, k, tau, "masked pieces")
    x[n - 1] = -float("inf")
    check_top(P, x, k, tau, "a row of nothing")
    if k <= 40:  # the loss takes the sum's logarithm: the teacher is the student, so the loss is 0 up to its rounding
        z = x[: n - 1].contiguous()
        val, idx, lse = (torch.zeros(n - 1, k, device="cuda"), torch.zeros(n - 1, k, dtype=torch.int32, device="cuda"),
                         torch.zeros(n - 1, device="cuda"))
        P.psw_top_logits(z, val, idx, temperature=tau, lse=lse)
        row = torch.zeros(n - 1, device="cuda")
        P.psw_distill(z, idx, val, row_loss=row, t_lse=lse, temperature=tau)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(row).all())


@pytest.mark.parametrize("tail", [False, True], ids=["entries", "rest"])
@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,k", [(6, 50, 7), (4, 900, 64), (3, 40000, 60), (3, 140000, 60)])
def test_labels_alone(P, n, c, k, type_, tail):
    """alpha 1: the loss is the label's, whatever the teacher says of classes that the student masks."""
    print(f"labels alone {n}x{c} k {k} {type_} rest={tail}", flush=True)
    rng = np.random.default_rng(c)
    z = rng.standard_normal((n, c)) * 2
    z[0, : c // 2] = -np.inf
    z[1, 5] = -np.inf
    x, _ = matrix(z, type_)
    z = x.double().cpu().numpy()
    idx = np.tile(np.arange(k, dtype=np.int32), (n, 1))
    val = rng.standard_normal((n, k)).astype(np.float32)
    lse = np.full(n, 6.0, np.float32)
    val[2, 1], lse[2] = np.nan, np.inf
    label = rng.integers(c // 2, c, n).astype(np.int32)
    weight = rng.uniform(0.5, 2, n).astype(np.float32)
    dz, _ = matrix(np.full((n, c), 7.0), type_)
    got = run(P, x, idx, val, lse if tail else None, label, weight, 3.0, 1.0, dz)
    val[2], lse[2] = 0.0, 6.0
    idx[:] = -1  # the formulas without their first terms
    ref = distill_ref(z, idx, val, None, label, weight.astype(np.float64), 3.0, 1.0)
    check_distill(got, dz, ref, weight.astype(np.float64), type_, "alpha 1")


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("n,c,gap", [(5, 100, 0), (4, 1003, 5), (3, 40000, 1), (2, 70001, 3)])
def test_gradients_beside_logits(P, n, c, gap, type_):
    """Logits and gradients as columns of one matrix, either first; nothing else is written."""
    print(f"beside {n}x{c} gap {gap} {type_}", flush=True)
    rng = np.random.default_rng(c)
    tau, alpha = 2.0, 0.3
    label, weight = rng.integers(0, c, n).astype(np.int32), rng.uniform(0.5, 2, n).astype(np.float32)
    for first in (True, False):
        both = torch.full((n, 2 * c + 2 * gap), 7.0, dtype=TYPES[type_], device="cuda")
        left, right = both[:, :c], both[:, c + gap:2 * c + gap]
        x, d = (left, right) if first else (right, left)
        x.copy_(torch.from_numpy(rng.standard_normal((n, c)) * 3))
        z = x.double().cpu().numpy()
        idx, val, lse = teacher(rng, z, 7, tau, "odd")
        got = run(P, x, idx, val, lse, label, weight, tau, alpha, d)
        ref = distill_ref(z, idx, val, lse.astype(np.float64), label, weight.astype(np.float64), tau, alpha)
        check_distill(got, d, ref, weight.astype(np.float64), type_, "beside")
        assert np.array_equal(x.double().cpu().numpy(), z)
        assert bool((both[:, c:c + gap] == 7).all()) and bool((both[:, 2 * c + gap:] == 7).all())
