"""A workspace for the largest chunk has room for every smaller one's own number of pieces (host only)."""
import pytest

import paper_2605_17757_amd as ok


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("n_q,B,Hq,Hkv,mp", [
    (8192, 1, 32, 8, 256), (8192, 1, 32, 8, 2048), (4096, 1, 64, 8, 512), (2048, 16, 64, 8, 512), (5000, 3, 7, 1, 300),
    (3000, 2, 16, 1, 1024), (700, 64, 32, 8, 512), (40, 1, 4, 4, 100), (1, 1, 32, 8, 2048), (100, 4, 32, 8, 1000),
    (6000, 1, 1, 1, 16384)])
def test_one_workspace_keeps_smaller_chunks_pieces(quantized, n_q, B, Hq, Hkv, mp):
    lay = ok.Layout(Hkv, 1000)
    whole = ok.chunk_workspace_bytes(lay, n_q, B, Hq, mp, 0, quantized)
    step = max(1, n_q // 2000)
    for n in sorted({*range(1, min(n_q, 600) + 1), *range(1, n_q + 1, step), n_q}):
        s = ok.chunk_default_splits(lay, n, B, Hq, mp)
        need = ok.chunk_workspace_bytes(lay, n, B, Hq, mp, s, quantized)
        assert need <= whole, "%d tokens in %d pieces need %d bytes of %d" % (n, s, need, whole)


def test_sizes_grow_with_the_chunk():
    lay = ok.Layout(8, 1000)
    for quantized in (False, True):
        last = 0
        for n in (1, 2, 8, 9, 64, 128, 129, 512, 1024, 4000, 8192, 20000):
            size = ok.chunk_workspace_bytes(lay, n, 1, 32, 512, 0, quantized)
            assert size >= last
            last = size


def test_an_explicit_number_of_pieces_is_sized_as_it_is():
    lay = ok.Layout(8, 1000)
    assert ok.chunk_workspace_bytes(lay, 8192, 1, 32, 256, 1, False) == 256
    assert ok.chunk_workspace_bytes(lay, 0, 1, 32, 256, 0, False) == 256
