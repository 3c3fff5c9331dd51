"""Arguments that the attention layers' binding refuses on a machine with a
device: what is no tensor, or has no dimensions."""
import pytest
import torch

import paper_2609_30950_amd as K

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [None, 3, [1, 2], torch.tensor(1)], ids=str)
def test_no_tensor_or_no_dimensions(bad):
    pages = K.Pages(2, 64, 8, 4)
    t = torch.zeros(2, device="cuda", dtype=torch.int32)
    cfg, lat = K.AttnConfig(pages, 4, 2, 64), K.LatentConfig(pages, 4, 64, 32, 256, 64)
    kc, vc = K.new_attn_caches(cfg)
    with pytest.raises(K.KdaError):
        K.kda_pages_plan(pages, t, t, t[:1], t, t, t, t[:1], t, bad, t)
    with pytest.raises(K.KdaError):
        K.kda_attn_append(cfg, bad, bad, bad, kc, vc)
    with pytest.raises(K.KdaError):
        K.kda_latent_append(lat, bad, bad, bad, K.new_latent_cache(lat))
    with pytest.raises(K.KdaError):
        K.kda_latent_prefill(lat, 100, bad, bad, t, t, t, t, t, t, t, t)
    with pytest.raises(K.KdaError):
        K.kda_attn_step(cfg, bad, kc, vc, t, t, t, bad)
    with pytest.raises(K.KdaError):
        K.kda_latent_step(lat, bad, bad, t, t, t, t, t, t, bad)
