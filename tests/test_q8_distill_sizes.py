"""Sizes of the 8-bit products, the top logits and the distillation loss at the edges of their rules: host checks alone, so
that every call here returns before a kernel would start."""
import pytest


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
