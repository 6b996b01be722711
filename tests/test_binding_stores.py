"""Codes and scales as the binding takes them, without a GPU: which slices of larger buffers have usable pitches."""
import pytest
import torch

from paper_1905_05686_amd import binding


def _bytes(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


@pytest.mark.parametrize("block_bytes", [16, 32])
@pytest.mark.parametrize("cols", [1, 32, 33, 96, 100, 129, 400])
@pytest.mark.parametrize("rows", [1, 2, 5])
def test_slices(rows, cols, block_bytes):
    """The first rows and blocks of buffers with whole pitches; one row of them has whole pitches too, whatever its stride says."""
    blocks = -(-cols // 32)
    codes, scales = _bytes(9, block_bytes * blocks + 48), _bytes(9, blocks // 4 * 4 + 8)
    for c, s in ((codes[:rows], scales[:rows]), (codes[:rows, :block_bytes * blocks], scales[:rows, :blocks]),
                 (codes[4:4 + rows, :block_bytes * blocks], scales[4:4 + rows, :blocks])):
        cp, ldc, sp, lds = binding._store(-1, (c, s), rows, cols, block_bytes)
        assert (cp, sp) == (c.data_ptr(), s.data_ptr())
        assert ldc % 16 == 0 and ldc >= block_bytes * blocks and lds % 4 == 0 and lds >= blocks
        assert rows == 1 or (ldc, lds) == (c.stride(0), s.stride(0))


def test_a_single_row_of_any_stride():
    codes, scales = _bytes(64), _bytes(8)
    for c in (codes[:16].unsqueeze(0), codes[:16].as_strided((1, 16), (0, 1)), codes[:16].as_strided((1, 16), (1, 1))):
        for s in (scales[:1].unsqueeze(0), scales[:1].as_strided((1, 1), (0, 1)), scales[:4].unsqueeze(0)):
            _, ldc, _, lds = binding._store(-1, (c, s), 1, 20, 16)
            assert (ldc, lds) == (16, 4)
