"""Bytes of the token heads' workspace, from the host alone (CPU)."""
import pytest
import torch  # before the library: both then share one HIP runtime

PIECE = 1 << 30


def size(lib, shapes, d, f32=False, dh=False):
    """Workspace of tenants of (targets, vocabulary), without row gradients; nothing reads what the addresses name."""
    from paper_2607_16074_amd import _abi
    import ctypes as C
    G = len(shapes)
    heads, ios = (_abi.jn_token_head * G)(), (_abi.jn_token_io * G)()
    for h, io, (n, v) in zip(heads, ios, shapes):
        h.vocab, h.W, io.n, io.dw_f32 = v, 4096, n, int(f32)
        for f in ("rows", "targets", "logp", "loss", "dW"):
            setattr(io, f, 4096)
        io.dh = 4096 if dh else None
    b = C.c_size_t()
    assert lib._lib.jn_tokens_workspace_size(d, heads, ios, G, C.byref(b)) == 0
    return b.value


@pytest.mark.parametrize("case", [([(5447, 200000)], 128), ([(5000, 120000)], 128), ([(3000, 250000)], 256),
                                  ([(8192, 160001)], 2048), ([(1 << 20, 1000)], 64), ([(1 << 20, 300), (1 << 20, 5000)], 64),
                                  ([(700000, 513), (700001, 400)], 64), ([(20000, 90001)] * 5 + [(40000, 260)] * 20, 64),
                                  ([(500000, 700), (300, 1 << 24)], 128), ([(2000, 300007), (0, 77), (31, 70)], 64)],
                         ids=lambda c: "-".join(f"{n}x{v}" for n, v in c[:3]) if isinstance(c, list) else str(c))
def test_the_kept_piece_is_within_its_bytes(lib, case):
    """What is there beside it: gathered rows, 32 bytes an entry, a part of 8 bytes for every 32 columns of an entry at
    most (an even number of parts), the table."""
    shapes, d = case
    rest = sum(n * (2 * d + 32 + 8 * ((v + 63) // 64 * 2 + 4)) for n, v in shapes) + 4096 * (len(shapes) + 4)
    # a grouped call's pieces: their problems and descriptors
    rest += len(shapes) * (200 + 600 * 64)
    assert size(lib, shapes, d) <= PIECE + rest


@pytest.mark.parametrize("dh", [False, True], ids=["w", "wh"])
@pytest.mark.parametrize("case", [(1, 160001, 2048), (16, 160001, 2048), (17, 160001, 2048), (64, 160001, 2048),
                                  (64, 4000001, 64), (64, 4300001, 64), (16, 1 << 24, 64), (33, 1 << 24, 64), (1, 1 << 24, 8192)],
                         ids=lambda c: "-".join(map(str, c)))
def test_calls_of_few_entries(lib, case, dh):
    """All logits in fp32 for 16, 32 or 64 entries of a vocabulary row, with dh as many bytes again; no more than a piece.
    dh's sums: two fp32 rows an entry for every range of at least 512 columns, 512 ranges at most, or one of 2^31 bytes
    of W."""
    n, v, d = case
    wide = (16 if n <= 16 else 32 if n <= 32 else 64) * (8 if dh else 4) * v
    planes = 2 * 4 * n * d * (min(512, (v + 511) // 512) + 2 * v * d // (1 << 31) + 2) if dh else 0
    got = size(lib, [(n, v)], d, False, dh)
    parts = 8 * n * 514 + (1 << 20)
    if wide <= PIECE:
        assert got <= wide + planes + parts + n * (2 * d + 32)
    assert got <= PIECE + planes + n * (2 * d + 32) + max(parts, 8 * n * (v // 32 + 4)) + (1 << 20)
