"""What a pipeline with sampling would fail on after its prefill is refused when it is made."""
from types import SimpleNamespace

import pytest
import torch

from paper_2405_14371_b200.pipeline import ShardPipeline


def _pipeline(sampling, batch=4):
    stream = SimpleNamespace(cuda_stream=1, device=torch.device("cpu"))
    shards = [SimpleNamespace(stream=stream, layer_end=2, desc=SimpleNamespace(n_layers_total=2))]
    return ShardPipeline(shards, [[0] * batch, [1] * batch], batch, "sequential", sampling=sampling)


def test_settings_of_another_type_layout_or_device_are_refused():
    u, t, k = torch.rand(3, 2, 4), torch.ones(2, 4), torch.ones(2, 4, dtype=torch.int32)
    _pipeline({"u": u, "temperature": t, "top_p": t, "min_p": t, "top_k": k})
    _pipeline({"u": torch.rand(3, 2, 9)[..., :4], "top_k": torch.ones(2, 8, dtype=torch.int32)[:, 2:6]})      # spaced rows serve
    _pipeline({"u": torch.rand(1, 2, 3)[..., ::3], "temperature": torch.ones(2, 2)[:, ::2]}, batch=1)
    for bad in ({"u": u.double()}, {"u": u, "top_k": t}, {"u": u, "top_k": k.long()}, {"u": u, "temperature": t.half()}, {"u": u, "min_p": k},
                {"u": torch.rand(3, 2, 8)[..., ::2]}, {"u": u, "top_p": torch.ones(4, 2).t()}, {"u": u, "top_p": torch.ones(2, 1).expand(2, 4)},
                {"u": u, "temperature": t.to("meta")}, {"u": u.to("meta")}, {"u": u[:0]}):
        with pytest.raises(ValueError):
            _pipeline(bad)
