"""Tiles of the vocabulary loss, seen from the host: the forward's workspace
holds two floats per row and column tile, so its size tells the tile's width."""

import pytest

from paper_2607_02805_gb300 import binding as b


def up(x, m):
    return (x + m - 1) // m * m


def tile_columns(rows, d_model, vocab, dtype):
    """Bounds of the tile width: tiles = ceil(vocab / width)."""
    r = up(rows, 256)
    n = b.bdscan_lm_loss_forward_workspace_size(b.make_lm_loss_dims(rows, d_model, vocab, dtype))
    pieces = 3 if dtype == b.BDSCAN_F32 else 1
    n -= 256 + 5 * up(4 * r, 256) + up(r * d_model * 2 * pieces, 256) + up(4 * r, 256)  # the rows that count
    if pieces == 3:
        n -= up(vocab * d_model * 2 * pieces, 256)  # w in pieces
    tiles, rest = divmod(n, 8 * r)
    assert rest == 0 and tiles > 0
    return vocab / tiles


@pytest.mark.parametrize("d_model,vocab", [(448, 50048), (832, 50304), (1664, 50304)])
def test_blocks_of_rows_are_planned_for_all_of_them(d_model, vocab):
    """More than 128 rows may all count: tiles of single CTAs (128 rows, up to 128 columns) read every row of w twice
    then, pairs (256 rows) once. Whether that is better must not be decided by what one caller's masks leave."""
    for rows in (200, 256):
        assert tile_columns(rows, d_model, vocab, b.BDSCAN_BF16) > 128
    assert tile_columns(128, d_model, vocab, b.BDSCAN_BF16) <= 128


def test_pieces_of_the_backward_fill_their_limit():
    """The gradient at the logits of 16384 rows over 16384 entries is 512 MiB in bf16, which is one piece."""
    rows, d_model, vocab = 16384, 448, 16384
    n = b.bdscan_lm_loss_backward_workspace_size(b.make_lm_loss_dims(rows, d_model, vocab, b.BDSCAN_BF16))
    n -= 256 + 5 * 4 * rows + 2 * rows * d_model * 2  # the rows that count, their h and its scaled copy
    assert 1 << 29 <= n <= (1 << 29) + (64 << 20)
    n = b.bdscan_lm_loss_backward_workspace_size(b.make_lm_loss_dims(rows, d_model, vocab + 1, b.BDSCAN_BF16))
    assert n < 1 << 29  # two pieces of half the size
