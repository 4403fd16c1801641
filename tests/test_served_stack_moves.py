"""The angles of a served stack follow its weights to another device and keep their type."""
import copy

import torch

from paper_2506_17870_b200.attention import DecoderStack, rotary_angles


def stack(device="cpu"):
    return DecoderStack(1, 64, 64, 1, 1, 64, positions=33, device=device)


def test_to_another_device():
    moved = stack().to("meta")
    assert moved.angles.is_meta and moved.final_weight.is_meta and moved.angles.shape == (33, 64)


def test_angles_of_ones_own_stay():
    s = stack()
    s.angles = rotary_angles(50, 64, base=1e6, device="cpu")
    assert torch.equal(s.to("cpu").angles, rotary_angles(50, 64, base=1e6, device="cpu")) and torch.equal(copy.deepcopy(s).angles, s.angles)


def test_another_type():
    assert stack().double().angles.dtype is torch.float32


def test_from_no_device():
    s = stack("meta").to_empty(device="cpu")
    assert torch.equal(s.angles, rotary_angles(33, 64, device="cpu"))
