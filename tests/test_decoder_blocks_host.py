"""Host-side check of the decoder's number of blocks (no GPU)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2209_04161_amd import decoder  # noqa: E402


def test_a_decoder_without_blocks_is_refused():
    """Its result would be that of the last norm's first row."""
    lut = torch.zeros(1 << 14, dtype=torch.int32)
    for blocks in (0, -1):
        with pytest.raises(ValueError):
            decoder.Decoder(blocks, 32, 2, 1, 32, lut, 7)
    assert len(decoder.Decoder(1, 32, 2, 1, 32, lut, 7).blocks) == 1
