"""The rotary frequencies of a DynamicMaskAttention: a buffer in fp32 that moves with the module and changes neither its values nor, where it stays
on its device, its place in memory."""
import copy

import pytest
import torch

from paper_2508_02124_amd.torch_api import DynamicMaskAttention, rotary_freqs


def module(**more):
    return DynamicMaskAttention(4, 2, 64, 8, **{**dict(rotary_dim=32, rotary_base=500.0), **more})


STAY = {"float": lambda m: m.float(), "bfloat16": lambda m: m.bfloat16(), "double": lambda m: m.double(), "half": lambda m: m.half(), "cpu": lambda m: m.cpu(),
        "to": lambda m: m.to("cpu", torch.bfloat16), "there and back": lambda m: m.bfloat16().float(),
        "inside another": lambda m: torch.nn.Sequential(m).to(torch.float64), "apply": lambda m: m._apply(lambda t: t.clone())}


@pytest.mark.parametrize("how", STAY)
def test_frequencies_of_one_s_own_stay(how):
    """Set in place, or put in the buffer's place (scaled, for longer contexts)."""
    for put in (lambda m, f: m.rotary_freqs.copy_(f), lambda m, f: setattr(m, "rotary_freqs", f)):
        m, own = module(), rotary_freqs(32, 500.0) / 8
        put(m, own)
        held, place = m.rotary_freqs, m.rotary_freqs.data_ptr()
        STAY[how](m)
        assert m.rotary_freqs is held and m.rotary_freqs.data_ptr() == place
        assert torch.equal(m.rotary_freqs, own) and m.rotary_freqs.dtype == torch.float32


def test_copies_and_modules_without():
    m = module()
    m.rotary_freqs.mul_(0.25)
    other = copy.deepcopy(m).bfloat16()
    assert torch.equal(other.rotary_freqs, rotary_freqs(32, 500.0) / 4) and other.rotary_freqs is not m.rotary_freqs
    plain = module(rotary_dim=0).bfloat16()
    assert plain.rotary_freqs is None and plain.W.dtype == torch.bfloat16


def test_a_module_without_values_gets_those_of_its_base():
    m = module(device="meta")
    assert m.rotary_freqs.is_meta
    m.to_empty(device="cpu")
    assert torch.equal(m.rotary_freqs, rotary_freqs(32, 500.0))
    there = module()
    there.rotary_freqs.mul_(0.5)
    assert there.to("meta").rotary_freqs.is_meta                     # (values are gone from here on)


@pytest.mark.gpu
def test_frequencies_of_one_s_own_move(gpu):
    """To the device and back; there, calls that change nothing leave the buffer where a captured graph reads it."""
    m, own = module(), rotary_freqs(32, 500.0) / 8
    m.rotary_freqs.copy_(own)
    m.to(gpu)
    held, place = m.rotary_freqs, m.rotary_freqs.data_ptr()
    assert held.device == gpu and torch.equal(held.cpu(), own)
    for again in (lambda: m.to(gpu), lambda: m.cuda(), lambda: m.float(), lambda: m.bfloat16(), lambda: m.float()):
        again()
        assert m.rotary_freqs is held and held.data_ptr() == place and held.dtype == torch.float32
    m.bfloat16().cpu()
    assert torch.equal(m.rotary_freqs, own) and m.rotary_freqs.dtype == torch.float32
    m.to(gpu, torch.float16)
    assert torch.equal(m.rotary_freqs.cpu(), own)
