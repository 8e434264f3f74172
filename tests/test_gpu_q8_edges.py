"""8-bit operands and products at the ends of their range, what the 8-bit instruction drops, and column
sums of one rounding."""
import numpy as np
import pytest
import torch

from tests import q8_ref
from tests.test_gpu_q8 import TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_1912_12675_amd import psw
    psw.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return psw


LOWEST = {"f32": -3.4028234663852886e38, "bf16": -3.3895313892515355e38}


def stands_for(pair, tiles):
    """The numbers of an operand's bytes, in 64 bits."""
    q, s = (t.cpu().numpy() for t in pair)
    wide = np.repeat(s[:, : q.shape[1] // 128].astype(int) - 127, 128, axis=1)
    if tiles:
        wide = np.repeat(wide, 128, axis=0)[: len(q)]
    return np.ldexp(q8_ref.decode(q), wide)


@pytest.mark.parametrize("tiles", [False, True], ids=["rows", "tiles"])
@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 3), (5, 300), (130, 257)])
def test_largest_numbers(P, rows, cols, type_, tiles):
    """Finite numbers become finite ones, below 2^128, in every order and kernel."""
    print(f"largest numbers {rows}x{cols} {type_} tiles={tiles}", flush=True)
    rng = np.random.default_rng(rows)
    x = np.ldexp(rng.uniform(-1, 1, (rows, cols)), rng.integers(100, 129, (rows, cols)))
    x = np.clip(x, LOWEST[type_], -LOWEST[type_])
    x[0, 0] = LOWEST[type_]
    x[rows - 1, cols - 1] = -LOWEST[type_]
    x[rows // 2, cols // 3] = np.ldexp(247.0 if type_ == "bf16" else 247.99, 120)  # the largest that rounds to 240 * 2^120
    xt = torch.from_numpy(x.astype(np.float32)).cuda().to(TYPES[type_])
    x = xt.double().cpu().numpy()
    q, s = P.q8_operand(rows, cols, tiles)
    qt, st = P.q8_operand(cols, rows, tiles)
    P.psw_q8_quant(xt, q, s, qt, st, tiles=tiles)
    alone = P.q8_operand(rows, cols, tiles)
    P.psw_q8_quant(xt, *alone, tiles=tiles)
    torch.cuda.synchronize()
    assert torch.equal(q, alone[0]) and torch.equal(s, alone[1])
    for pair, m in (((q, s), x), ((qt, st), x.T)):
        ref_q, ref_e, _ = q8_ref.quantise(m, tiles)
        wide = np.repeat(np.repeat(ref_e, 128, axis=1), 128 if tiles else 1, axis=0)[: len(m)]
        ref = np.ldexp(ref_q, wide)
        assert (np.abs(ref) >= 2.0**128).any()  # the nearest: past every float
        ref = np.clip(ref, -240 * 2.0**120, 240 * 2.0**120)
        np.testing.assert_array_equal(stands_for(pair, tiles), ref)


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 20, 100])
def test_masked_inputs(P, n, type_):
    """Inputs of the type's lowest number under weights of 0 add nothing; under a tiny weight an ordinary number."""
    print(f"masked inputs {n} {type_}", flush=True)
    rng = np.random.default_rng(n)
    fin, out = 300, 70
    x = rng.standard_normal((n, fin))
    x[:, 128:200] = LOWEST[type_]
    w = rng.standard_normal((out, fin))
    w[:, 128:256] = 0.0
    w[:, 130] = 2.0**-120
    x8, w8 = P.q8_operand(n, fin), P.q8_operand(out, fin, True)
    P.psw_q8_quant(torch.from_numpy(x.astype(np.float32)).cuda().to(TYPES[type_]), *x8)
    P.psw_q8_quant(torch.from_numpy(w.astype(np.float32)).cuda(), *w8, tiles=True)
    y = torch.zeros(n, out, dtype=TYPES[type_], device="cuda")
    P.psw_fc8_fwd(x8, w8, fin, y)
    torch.cuda.synchronize()
    a, b = stands_for(x8, False), stands_for(w8, True)
    want, size, square = a @ b.T, np.abs(a) @ np.abs(b).T, np.sqrt((a * a) @ (b * b).T)
    # fp32: a step of 2^-23 for each addition; bfloat16: half a step, and seven times the 7e-5 of the root of the
    # products' squares that the 8-bit instruction was measured to drop
    bound = (fin + 8) * 2.0**-23 * size if type_ == "f32" else 2.0**-8 * np.abs(want) + (1 + 2.0**-8) * 2.0**-11 * square
    assert (np.abs(y.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("n", [16, 32, 256])
def test_exact_range(P, n):
    """One product a result, so that a float32 result is exact wherever the operand's element is a bfloat16 number: every
    e4m3 value at scales over their whole range, with value * scale from 2^-133 up to below 2^128.  Below, an element is off
    by at most half of 2^-133."""
    fin, out = 1024, 64
    for lo in (1, 9, 64, 124, 190, 240, 247):
        print(f"exact range {n} rows, scales from {lo}", flush=True)
        e = np.minimum(lo + np.arange(8), 254)
        down = -100 if lo >= 127 else 100
        w8 = torch.full((out, fin), 0x38, dtype=torch.uint8, device="cuda"), torch.full((1, 8), 127 + down, dtype=torch.uint8, device="cuda")
        s = torch.from_numpy(np.tile(e.astype(np.uint8), (n, 1))).cuda()
        for start in range(0, 256, n):
            for turn in range(8):
                m = np.arange(n)
                at = (m + turn) % 8
                v = ((start + m) % 256).astype(np.uint8)
                v[(v & 127) == 127] = 0
                for _ in range(16):  # an exponent less until the element is below 2^128
                    v = np.where(np.ldexp(np.abs(q8_ref.decode(v)), e[at] - 127) >= 2.0**128, v - 8, v).astype(np.uint8)
                q = np.zeros((n, fin), np.uint8)
                q[m, at * 128 + (37 * m + turn) % 128] = v
                y = torch.zeros(n, out, device="cuda")
                P.psw_fc8_fwd((torch.from_numpy(q).cuda(), s), w8, fin, y)
                torch.cuda.synchronize()
                element = np.ldexp(q8_ref.decode(v), e[at] - 127)
                off = np.abs(y.double().cpu().numpy() - np.ldexp(element, down)[:, None])
                whole = np.ldexp(element, 133) == np.round(np.ldexp(element, 133))  # numbers that bfloat16 has
                assert (off[whole] == 0).all(), (lo, element[whole][(off[whole] > 0).any(1)])
                assert (off <= 2.0**(down - 134)).all(), (lo, off.max())


@pytest.mark.parametrize("n,fin,out", [(20, 2000, 300), (64, 4096, 512), (128, 4096, 640), (700, 1024, 520), (2100, 512, 2050)])
def test_bfloat16_products_in_the_norm(P, n, fin, out):
    """Against the nearest bfloat16 numbers of the exact results.  The 8-bit instruction drops at most d = 7e-5 of the root
    of the summed squares (measured); a result so becomes the neighbouring number, a step of at most 2^-7 away, with
    probability d / step, which leaves a mean square of d step, and d^2 where the result is smaller than d.  Twice that
    for chance."""
    print(f"norm {n}x{fin}->{out}", flush=True)
    rng = np.random.default_rng(n)
    x8, w8 = P.q8_operand(n, fin), P.q8_operand(out, fin, True)
    P.psw_q8_quant(torch.from_numpy(rng.standard_normal((n, fin)).astype(np.float32)).cuda(), *x8)
    P.psw_q8_quant(torch.from_numpy(rng.standard_normal((out, fin)).astype(np.float32)).cuda(), *w8, tiles=True)
    y = torch.zeros(n, out, dtype=torch.bfloat16, device="cuda")
    P.psw_fc8_fwd(x8, w8, fin, y)
    torch.cuda.synchronize()
    a, b = torch.from_numpy(stands_for(x8, False)).cuda(), torch.from_numpy(stands_for(w8, True)).cuda()
    want, square = a @ b.t(), (a.square() @ b.square().t()).sqrt()
    d = 7e-5 * square
    off = (y.double() - want.to(torch.bfloat16).double()).square().sum()
    assert float(off) <= 2 * float((d * 2.0**-7 * want.abs() + d.square()).sum())


@pytest.mark.parametrize("type_", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 5), (128, 130), (129, 9), (1000, 257), (5000, 3)])
def test_column_sums_round_once(P, rows, cols, type_):
    """Column sums are formed in 64 bits from the first row on: fewer than rows + 40 additions, each off by at most
    half a step, 2^-53 of what is there, and one rounding to float32."""
    print(f"column sums {rows}x{cols} {type_}", flush=True)
    rng = np.random.default_rng(rows + cols)
    x = rng.standard_normal((rows, cols)) * np.exp(3 * rng.standard_normal((rows, cols)))
    if rows > 1:  # large numbers that cancel
        x[0, 0] = 2.0**30
        x[rows - 1, 0] = -(2.0**30)
        x[1:rows // 2 + 1, cols - 1] = -x[rows - rows // 2:, cols - 1][::-1]
    xt = torch.from_numpy(x.astype(np.float32)).cuda().to(TYPES[type_])
    x = xt.double().cpu().numpy().astype(np.longdouble)
    total = torch.zeros(cols, device="cuda")
    P.psw_q8_quant(xt, colsum=total)
    q = P.q8_operand(cols, rows)
    again = torch.zeros(cols, device="cuda")
    P.psw_q8_quant(xt, qt=q[0], st=q[1], colsum=again)
    torch.cuda.synchronize()
    assert torch.equal(total, again)
    want, size = x.sum(0), np.abs(x).sum(0)
    bound = 2.0**-24 * np.abs(want) + (1 + 2.0**-24) * (rows + 40) * 2.0**-53 * size + 2.0**-149
    assert (np.abs(total.double().cpu().numpy() - want) <= bound).all()
