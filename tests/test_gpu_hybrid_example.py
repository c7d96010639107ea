"""The example of a hybrid model: DeltaNet and attention layers over states and paged caches, in chunks and in one piece."""
import pytest

import example_hybrid

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layers,heads,head_size,window", [(4, 4, 64, 256), (2, 2, 128, 0), (4, 2, 128, 100)])
def test_chunks_give_what_one_piece_gives(layers, heads, head_size, window):
    """The same arithmetic on the same values up to bf16 roundings (2^-8 each, of every layer's operands, and an 8-bit number of a key or value that
    such a difference tips over, 2^-4 of that element): half a per cent per layer is several times what they add up to."""
    off, _ = example_hybrid.run(layers, heads, head_size, window, tokens=6)
    print("relative difference", off)
    assert off <= 5e-3 * layers
