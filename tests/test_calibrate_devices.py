"""Replays run on the device that their tensors are on, whichever is the current one; layers may lie on different devices."""
import contextlib

import numpy as np
import pytest
import torch

from paper_2605_17170_amd import calibrate


class Calls:
    """Stands for the device's entry points: notes the device that is the current one during each call."""

    def __init__(self, monkeypatch):
        self.current, self.seen = None, []
        monkeypatch.setattr(torch.cuda, "device", self.device)
        monkeypatch.setattr(calibrate.harness, "default_shared_units", lambda device=None: 256)
        for name in ("tkv_quantize_rows", "tkv_prefill_attention", "tkv_head_distortion"):
            monkeypatch.setattr(calibrate.tkv, name, lambda *a, _name=name, **kw: self.seen.append((_name, self.current)))

    @contextlib.contextmanager
    def device(self, device):
        before, self.current = self.current, torch.device(device)
        yield
        self.current = before


def inputs(n, device):
    return tuple(torch.zeros((n, h, 128), dtype=torch.bfloat16, device=device) for h in (4, 2, 2))


def test_calls_are_made_with_the_replays_device_as_the_current_one(monkeypatch):
    calls = Calls(monkeypatch)
    replay = calibrate.Replay([0, 5, 9], 4, 2, 0.1, "cpu", calibrate.tkv.TKV_KEYS_PER_CHANNEL)
    replay.distortion(*inputs(9, "cpu"), np.zeros(9, np.uint8), 0, 2)
    assert calls.seen == [(name, torch.device("cpu")) for name in ("tkv_quantize_rows", "tkv_prefill_attention", "tkv_head_distortion")]


@pytest.mark.parametrize("which", [0, 1, 2])
def test_tensors_of_another_device_are_refused(monkeypatch, which):
    calls = Calls(monkeypatch)
    replay = calibrate.Replay([0, 5, 9], 4, 2, 0.1, "cpu")
    tensors = list(inputs(9, "cpu"))
    tensors[which] = tensors[which].to("meta")
    with pytest.raises(ValueError):
        replay.attention(*tensors, np.zeros(9, np.uint8), replay.plain)
    assert not calls.seen


def test_layers_of_different_devices_have_replays_of_their_own(monkeypatch):
    made = []

    class Replay:
        def __init__(self, seq_indptr, n_q_heads, n_kv_heads, sm_scale, device, key_axis):
            self.device, self.plain, self.status = torch.device(device), "plain", torch.zeros(1, dtype=torch.int32)
            made.append(self)

        def attention(self, q, K, V, widths, out):
            assert q.device == K.device == V.device == self.device and out == "plain"

        def distortion(self, q, K, V, tags, tag, bits):
            assert q.device == self.device
            return torch.full((2, 4), 1.0 if bits == 2 else 0.25, dtype=torch.float64)

    monkeypatch.setattr(calibrate, "Replay", Replay)
    layers = [inputs(9, d) for d in ("cpu", "meta", "cpu", "meta")]
    N, D2, D4 = calibrate.tag_distortions(layers, np.full(9, 3, np.uint8), [0, 5, 9], 0.1)
    assert [r.device.type for r in made] == ["cpu", "meta"] and D2[3] == 4.0 and D4[3] == 1.0 and N[3] == 9
    made[1].status += 64
    monkeypatch.setattr(calibrate, "Replay", lambda *a: made[0] if torch.device(a[4]).type == "cpu" else made[1])
    with pytest.raises(RuntimeError):
        calibrate.tag_distortions(layers, np.full(9, 3, np.uint8), [0, 5, 9], 0.1)
