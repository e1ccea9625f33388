"""DeviceWeights8 on a device that is not the current one: everything it launches runs with its own device current.  No GPU: the context
and the calls are stand-ins that note the device."""
import contextlib

import torch

from paper_2609_25405_b200 import binding as B
from paper_2609_25405_b200 import synth


def test_everything_runs_on_the_weights_device(monkeypatch):
    now, seen = ["other"], []

    @contextlib.contextmanager
    def device(d):
        was, now[0] = now[0], d
        yield
        now[0] = was

    class Context:
        def __init__(self, *a):
            seen.append(("context", now[0]))

        def quant_rows(self, w, codes, scale, index=None, stream=None):
            assert codes.shape == w.shape and scale.shape == w.shape[:1]
            seen.append(("quant_rows", now[0]))

        def close(self):
            pass

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda d=None: seen.append(("synchronize", d)))
    monkeypatch.setattr(B, "Context", Context)
    monkeypatch.setattr(B, "pack_f16_", lambda t, stream=None: (seen.append(("pack", now[0])), t)[1])
    shape = synth.ModelShape("w8", 2, 64, 1, 1, 64, 128, 64)
    random = B.DeviceWeights8.random_on_device(shape, device="cpu")
    assert len(seen) == 1 + 4 * shape.L + 2 and {d for _, d in seen} == {"cpu"}
    assert all(random.layers[l].wqkv and random.layers[l].down_scale for l in range(shape.L))
    seen.clear()
    B.DeviceWeights8.from_synth(synth.Weights(shape, 0), device="cpu")
    assert len(seen) == 1 + 4 * shape.L + 2 and {d for _, d in seen} == {"cpu"}
    assert now == ["other"]
