"""Sizes of the 8-bit products, the top logits and the distillation loss at the edges of their rules: host checks alone, so
that every call here returns before a kernel would start."""
import pytest
import torch

NULL, SHAPE = -1, -2
F32, BF16 = 0, 1
P16 = 1 << 20  # an address that is never used


@pytest.fixture(scope="module")
def L():
    from paper_1912_12675_amd import psw
    return psw.lib()


def pieces(n, nbytes, k):
    """Of a row of nbytes: 1 up to 256 KB; 16 KB each, 64 KB for many rows or many entries to merge."""
    if nbytes <= 1 << 18:
        return 1
    small = -(-nbytes >> 14)
    return -(-nbytes >> 16) if n >= 128 or k > 128 or small * k > 8192 else small


def test_top_logits_workspace_holds_the_pieces(L):
    """k keys of 8 bytes, and a largest and a sum for each piece, whether rows begin on 16 bytes or inside (16 bytes
    more).  Around 8192 keys more bytes mean fewer pieces."""
    edges = {b // size + d for b in (1 << 18, *(16384 * s for s in range(17, 258, 3))) for size in (2, 4) for d in (-5, -1, 0, 1, 5)}
    edges |= {(1 << p) + d for p in range(16, 21) for d in (-1, 0, 1)}
    ks = sorted({1, 2, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256} | {8192 // s for s in range(33, 257, 7)})
    tried = 0
    for classes in sorted(c for c in edges if 256 <= c <= 1 << 20):
        for k in ks:
            for n in (1, 127, 128):
                need = L.psw_top_logits_ws_bytes(n, classes, k)
                for size in (2, 4):
                    for more in (0, 16):
                        p = pieces(n, classes * size + more, k)
                        assert p == 1 or need >= n * p * (8 * k + 8), (n, classes, k, size, more)
                        tried += p > 1
    assert tried > 10000


def answer(L, rc):
    return rc, L.psw_last_error().decode()


# sizes whose launch has 2^32 threads, and the largest that can be counted: those are refused for what else they lack
@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("cols,tiles,both,rows,fits", [
    (1, 0, 0, 2**27, 2**27 - 8),        # 256 threads for 32 blocks, four of a row
    (600, 0, 0, 2**26, 2**26 - 4),      # eight blocks of a row
    (1, 0, 1, 2**30, 2**30 - 128),      # 512 threads for 128 rows
    (1, 1, 0, 2**30, 2**30 - 128),
    (300, 1, 1, 2**29, 2796202 * 128)])
def test_quantise_threads(L, cols, tiles, both, rows, fits, type_):
    def call(rows, x):
        q = (P16, P16, P16, P16) if both else (P16, P16, None, None)
        return answer(L, L.psw_q8_quant(rows, cols, type_, x, cols, tiles, *q, None, None, 0, None))

    rc, words = call(rows, P16)
    assert rc == SHAPE and "too large" in words, (rc, words)
    rc, words = call(fits, None)
    assert rc == NULL and "required" in words, (rc, words)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,out,fits", [(1, 2**27, 2**27 - 16), (16, 2**28, 2**27 - 16), (40, 2**30, 2**30 - 512)])
def test_product_threads(L, n, out, fits, type_):
    """Few rows: 512 threads for 16 columns, above 16 rows 256 for 64."""
    def call(out, x):
        return answer(L, L.psw_fc8_fwd(n, 128, out, x, P16, P16, P16, None, 0, type_, P16, P16, 1 << 60, None))

    rc, words = call(out, P16)
    assert rc == SHAPE and "too large" in words, (rc, words)
    rc, words = call(fits, None)
    assert rc == NULL and "required" in words, (rc, words)


ROWS = [(10, 64), (2020, 256), (10000, 512)]  # float32 classes (twice as many of bfloat16) and a row's threads


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("classes,threads", ROWS)
def test_rows_of_logits(L, classes, threads, type_):
    c, n = classes * (1 + type_), 2**32 // threads

    def top(n, val):
        return answer(L, L.psw_top_logits(n, c, type_, P16, c, 5, 1.0, val, P16, None, P16, 1 << 60, None))

    def loss(n, ws):
        return answer(L, L.psw_distill(n, c, type_, P16, c, 5, P16, P16, None, None, None, 1.0, 0.0, P16, None, None, 0, ws, 1 << 60, None))

    for call in (top, loss):
        rc, words = call(n, P16)
        assert rc == SHAPE and "too many rows" in words, (rc, words)
        rc, words = call(n - 1, None)
        assert rc == NULL and ("required" in words or "workspace" in words), (rc, words)


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
def test_rows_in_pieces(L, type_):
    """2^20 classes: 4 or 2 MB and up to 16 bytes more, in 65 or 33 pieces of 512 threads (top logits), in 129 or 65 of 256
    (the loss)."""
    c, pieces = 1 << 20, 33 if type_ else 65
    for n, want in ((2**32 // (pieces * 512) + 1, SHAPE), (2**32 // (pieces * 512) - 1, NULL)):
        rc, words = answer(L, L.psw_top_logits(n, c, type_, P16, c, 256, 1.0, P16 if want == SHAPE else None, P16, None, P16,
                                               1 << 60, None))
        assert rc == want, (rc, words)
    pieces = 65 if type_ else 129
    for n, want in ((2**32 // (pieces * 256) + 1, SHAPE), (2**32 // (pieces * 256) - 1, NULL)):
        rc, words = answer(L, L.psw_distill(n, c, type_, P16, c, 5, P16, P16, None, None, None, 1.0, 0.0, P16, None, None, 0,
                                            P16 if want == SHAPE else None, 1 << 60, None))
        assert rc == want, (rc, words)


def test_sizes_past_31_bits(monkeypatch):
    """ctypes keeps the low bits of an integer: a size of 2^32 + 5 would be one of 5."""
    from paper_1912_12675_amd import psw

    monkeypatch.setattr(psw, "_here", lambda t, what: None)  # tensors without memory in the place of a device's
    monkeypatch.setattr(psw, "_fast", psw._CtypesOnly())
    many = 2**32 + 5

    def new(*shape, dtype=torch.float32):
        return torch.empty(*shape, dtype=dtype, device="meta")

    def op(rows, k, tiles=False):
        return psw.q8_operand(rows, k, tiles, device="meta")

    i32 = torch.int32
    for call in (lambda: psw.psw_q8_quant(new(many, 1), None, None, *op(1, many)),
                 lambda: psw.psw_q8_quant(new(1, many), colsum=new(many), ws=new(8)),
                 lambda: psw.psw_fc8_fwd(op(1, many), op(3, many, True), many, new(1, 3), ws=new(8)),
                 lambda: psw.psw_fc8_fwd(op(many, 1), op(3, 1, True), 1, new(many, 3), ws=new(8)),
                 lambda: psw.psw_fc8_bwd_data(op(1, many), op(3, many, True), many, new(1, 3), ws=new(8)),
                 lambda: psw.psw_fc8_bwd_weight(op(3, many), op(2, many), many, new(3, 2), ws=new(8)),
                 lambda: psw.psw_fc8_bwd_weight(op(many, 1), op(2, 1), 1, new(many, 2), ws=new(8)),
                 lambda: psw.psw_top_logits(new(many, 3), new(many, 2), new(many, 2, dtype=i32), ws=new(8)),
                 lambda: psw.psw_top_logits(new(2, 3), new(2, many), new(2, many, dtype=i32), ws=new(8)),
                 lambda: psw.psw_distill(new(many, 3), new(many, 2, dtype=i32), new(many, 2), new(1), ws=new(8)),
                 lambda: psw.psw_distill(new(2, 3), new(2, many, dtype=i32), new(2, many), new(1), ws=new(8))):
        with pytest.raises(ValueError, match="below 2.31"):
            call()


@pytest.mark.parametrize("type_", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,ld,ldd,at,fine", [  # dlogits `at` elements behind the logits, rows of 100
    (4, 200, 200, 100, True), (4, 200, 200, -100, True), (4, 250, 250, 120, True), (4, 250, 250, 350, True),
    (4, 250, 250, 150, True), (4, 250, 250, -350, True), (4, 200, 200, 0, True), (4, 100, 100, 400, True),
    (1, 100, 100, 100, True), (4, 100, 100, -400, True),
    (4, 200, 200, 99, False), (4, 200, 200, 101, False), (4, 250, 250, 151, False), (4, 250, 250, -151, False),
    (4, 200, 201, 100, False), (4, 201, 200, -100, False), (4, 100, 100, 100, False), (4, 250, 250, 250, False),
    (1, 100, 100, 99, False), (4, 100, 100, 399, False)])
def test_gradients_beside_logits(L, n, ld, ldd, at, fine, type_):
    """Columns of one matrix do not overlap, however their rows lie."""
    z = P16
    dz = z + at * (2 if type_ == BF16 else 4)
    rc, words = answer(L, L.psw_distill(n, 100, type_, z, ld, 5, P16, P16, None, None, None, 1.0, 0.0, P16, None, dz, ldd, None,
                                        0, None))
    assert (rc == NULL and "workspace" in words) if fine else (rc == SHAPE and "overlaps" in words), (rc, words)
