"""The random numbers of hybrid_decode's positions, on the host: a sequence
that would need more of them than there are is refused before any device
work."""
import numpy as np
import pytest

from paper_2607_06763_amd import decode_sim as D
from paper_2607_06763_amd import hybrid_decode as H


def chain(n):
    return D.Tree(tokens=[1] * n, parent=[i - 1 for i in range(n)], ctx=[])


@pytest.mark.parametrize("layers", [("gdn",), ("gdn", "attn")])
def test_steps_past_the_last_number(layers):
    m = H.HybridModel(layers=layers, positions=16)
    dec = H.Decoder(m, 2, 8, np.zeros((2, 6), np.float32), max_pages=2, device="cpu")
    dec.prompt([[1], [2]])
    # the token after a node at depth 5 has position 6
    with pytest.raises(ValueError, match="random number"):
        dec.step([chain(3), chain(6)])
    # with enough of them the step goes on to the device calls, which refuse host tensors
    with pytest.raises(ValueError, match="device tensor"):
        dec.step([chain(3), chain(5)])


@pytest.mark.parametrize("shape", [(3, 16), (2,), (2, 16, 1), (16, 2)])
def test_shape_of_the_numbers(shape):
    m = H.HybridModel(positions=16)
    with pytest.raises(ValueError, match="u"):
        H.Decoder(m, 2, 8, np.zeros(shape, np.float32), max_pages=2, device="cpu")
