"""A model whose logits are all NaN, or all -inf, has no token to emit: the decode loop says so."""
import numpy as np
import pytest

from paper_2607_06763_amd import decode_sim as D
from paper_2607_06763_amd import hybrid_decode as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", [np.nan, -np.inf])
def test_no_token(what):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    m = H.HybridModel(layers=("gdn", "attn"), positions=64)
    dec = H.Decoder(m, 2, 8, np.full((2, 64), 0.5, np.float32), max_pages=4)
    dec.prompt([[1, 2], [3, 4, 5]])
    trees = [D.build_tree_best_first(m, p, budget=8) for p in ([1, 2], [3, 4, 5])]
    emitted = dec.step(trees)
    assert all(0 <= t < m.V for e in emitted for t in e)
    dec.unembed.fill_(what)
    with pytest.raises(RuntimeError, match="no token"):
        dec.step([D.build_tree_best_first(m, e, budget=8) for e in emitted])
