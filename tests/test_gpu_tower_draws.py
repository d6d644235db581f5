"""The random streams of a tower: no two of its parts draw under one key."""
import pytest

pytestmark = pytest.mark.gpu


def test_seeds_differ():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2010_11305_amd.tower import Tower

    t = Tower((64, 48, 33, 16), seed=9)
    seeds = [t.opt.seed, *(layer.seed for layer in t.layers), *(layer.weight_seed for layer in t.layers)]
    assert len(set(s % 2**64 for s in seeds)) == 7
