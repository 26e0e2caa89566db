"""The built-in choice of a product's way on 8-bit floats (host code, no GPU): the sizes that the GPU tests run every way at
(``f8_ways``) take the way that they are there for."""
import pytest

import f8_ways

cnn = pytest.importorskip("paper_1511_07376_amd.cnn", reason="libcnn.so not built")


@pytest.mark.parametrize("key", f8_ways.ROWS, ids=str)
def test_rows(key):
    for n, i, o in f8_ways.ROWS[key]:
        w = f8_ways.way(cnn, n, i, o)
        assert w.rows and (w.tokens, w.outs) == key
        assert cnn.lib.cnn_fc_f8_workspace_bytes(n, i, o) == 0
    assert any(i % 4 for _, i, _ in f8_ways.ROWS[key]) or key == (4, 1)


@pytest.mark.parametrize("key", f8_ways.TILES, ids=str)
def test_tiles(key):
    for n, i, o in f8_ways.TILES[key]:
        w = f8_ways.way(cnn, n, i, o)
        assert not w.rows and (w.tile_outs, w.tile_tokens, w.parts > 1) == key
        blocks = -(-i // 128)
        assert -(-blocks // w.run) == w.parts and (w.parts == 1 or w.run % 4 == 0)
        assert cnn.lib.cnn_fc_f8_workspace_bytes(n, i, o) == (4 * w.parts * n * o if w.parts > 1 else 0)
    whole = {i % 128 == 0 for _, i, _ in f8_ways.TILES[key]}
    assert whole == ({True} if key[0] == 256 else {True, False})


@pytest.mark.parametrize("n,i,o", [(1, 4096, 4096), (1, 9216, 8192), (1, 28672, 8192), (16, 4096, 4096)])
def test_few_tokens_stream_the_weights(n, i, o):
    assert f8_ways.way(cnn, n, i, o).rows


@pytest.mark.parametrize("n,i,o", [(1, 8192, 28672), (1, 4096, 128256), (64, 9216, 4096), (2048, 9216, 4096)])
def test_many_outputs_or_tokens_take_tiles(n, i, o):
    assert not f8_ways.way(cnn, n, i, o).rows
