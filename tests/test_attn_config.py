"""The attention layers' config objects (no GPU needed)."""
import copy
import pickle

import pytest
import torch

import paper_2609_30950_amd as K

PAGES = K.Pages(B=2, page=64, n_pages=8, max_pages=4)


@pytest.mark.parametrize("cfg", [PAGES, K.AttnConfig(PAGES, 4, 2, 64, dtype="f16", cache="e4m3", scale=0.3),
                                 K.LatentConfig(PAGES, 4, 128, 64, 512, 128)], ids=lambda c: type(c).__name__)
def test_configs_are_copied_and_sent(cfg):
    class Layer(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.cfg = cfg

    for other in (copy.copy(cfg), copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg)), copy.deepcopy(Layer()).cfg,
                  copy.deepcopy([cfg, cfg])[1]):
        assert other == cfg and type(other) is type(cfg) and bytes(other._c) == bytes(cfg._c)
        assert other._ref is not cfg._ref
        for name in ("key_shape", "value_shape", "cache_shape", "_need", "_t"):
            assert getattr(other, name, None) == getattr(cfg, name, None)
        if hasattr(other, "pages"):
            assert other.pages == PAGES


W = 2**32


@pytest.mark.parametrize("make", [
    lambda: K.Pages(W + 2, 64, 8, 4), lambda: K.Pages(2, W + 64, 8, 4), lambda: K.Pages(2, 64, W + 8, 4),
    lambda: K.Pages(2, 64, 8, W + 4), lambda: K.AttnConfig(PAGES, W + 4, 2, 64),
    lambda: K.AttnConfig(PAGES, 4, W + 2, 64), lambda: K.AttnConfig(PAGES, 4, 2, W + 64),
    lambda: K.LatentConfig(PAGES, W + 4, 128, 64, 512, 128), lambda: K.LatentConfig(PAGES, 4, 128, W + 64, 512, 128),
    lambda: K.LatentConfig(PAGES, 4, 128, 64, W + 512, 128), lambda: K.LatentConfig(PAGES, 4, 128, 64, 512, 128 - W),
    lambda: K.new_latent_prefill_workspace(K.LatentConfig(PAGES, 4, 128, 64, 512, 128), W + 100, device="cpu"),
    lambda: K.new_latent_prefill_workspace(K.LatentConfig(PAGES, 4, 128, 64, 512, 128), 2**31, device="cpu")])
def test_numbers_past_32_bits_are_refused(make):
    with pytest.raises(K.KdaError):
        make()
