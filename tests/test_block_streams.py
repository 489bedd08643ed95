"""Random words of different purposes under one seed: what the header says about them."""
import os

import numpy as np

import block_reference as ref
from conftest import ROOT


def test_layers_and_purposes_share_words_under_one_seed():
    """A dropout mask's 16-bit fields are the halves of the words that AdamW's rounding of tensor `layer` and the probes of
    direction `layer` draw in the same step: a seed for each purpose, as soma_drop's description asks for."""
    seed, t, layer, p = 0x1234567890ABCDEF, (3 << 32) + 11, 5, 0.25
    key = (seed & 0xFFFFFFFF, (seed >> 32) ^ (t >> 32))
    blocks = np.arange(64, dtype=np.uint64)
    counter = np.stack([blocks, np.full_like(blocks, layer), np.full_like(blocks, t & 0xFFFFFFFF), blocks >> np.uint64(32)], 1)
    words = ref.philox(counter, key).reshape(-1)                        # of elements 4 b .. of a tensor, of quad b
    fields = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 1).reshape(1, -1)
    assert np.array_equal(ref.keep(1, fields.shape[1], p, seed, t, layer) != 0, fields >= round(p * 65536))
    other = ref.keep(1, fields.shape[1], p, seed + 1, t, layer) != 0
    assert 0.5 < (other == (fields >= round(p * 65536))).mean() < 0.75  # 0.625 where nothing is shared
    with open(os.path.join(ROOT, "include", "soma.h")) as f:
        text = " ".join(f.read().replace("*", " ").split())
    assert "What a program draws for different purposes needs a seed for each" in text
    assert "a program that draws those too takes another seed here" in text
