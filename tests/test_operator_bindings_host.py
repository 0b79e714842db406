"""What the torch bindings of the transformer operators say to tensors, bands and numbers that do not fit, on the CPU: everything here is refused
in front of the library's launch. (The current device is told to be the CPU's, -1, for the checks to get as far.)"""
import numpy as np
import pytest
import torch

from paper_2507_05829_amd import lop
from test_operators_host import BAND, attention_op, product_op, quantize_op, rope_op

BANDS = [(0, 1 << 32), (1 << 32, (1 << 32) + 5), (0, (1 << 32) + 5), (0, 1 << 31), (-(1 << 32), 5), (-(1 << 40), -(1 << 40) + 3), (-1, 3), (np.int64(0), np.int64(1 << 33))]


@pytest.mark.parametrize("rows", BANDS, ids=str)
@pytest.mark.parametrize("call,op", [(lop.lop_quantize_blocks, quantize_op), (lop.lop_rowwise_f8, product_op), (lop.lop_head_norm_rope, rope_op),
                                     (lop.lop_attention, attention_op), (lop.lop_attention_workspace, attention_op)], ids=lambda c: c.__name__)
def test_bands_of_more_than_32_bits_do_not_wrap(call, op, rows):
    with pytest.raises(lop.LopError) as e:
        call(op(), rows)
    assert e.value.code == BAND


def test_bands_of_numpy_numbers():
    for t in (np.int32, np.int64, np.uint8):
        lop.lop_quantize_blocks(quantize_op(), (t(7), t(7)))        # empty: nothing is enqueued
    with pytest.raises(TypeError):
        lop.lop_quantize_blocks(quantize_op(), (0.0, 5.0))


# ------------------------------------------------------------------ tensors


class Calls:
    """Arguments of each operator's call, by name, that fit."""

    def __init__(self):
        f8, b16, i32 = torch.float8_e4m3fn, torch.bfloat16, torch.int32
        zeros = torch.zeros
        self.of = {
            "quantize_blocks": dict(x=zeros(3, 128, dtype=b16), q=zeros(3, 128).to(f8), scale=zeros(3, 1)),
            "rowwise_f8": dict(x=zeros(3, 128).to(f8), x_scale=zeros(3, 1), w=zeros(5, 128).to(f8), w_scale=zeros(1, 1), bias=zeros(5), residual=zeros(3, 5, dtype=b16),
                               y=zeros(3, 5, dtype=b16)),
            "head_norm_rope": dict(q=zeros(3, 2, 64, dtype=b16), k=zeros(3, 1, 64, dtype=b16), positions=zeros(3, dtype=i32), freq=zeros(32), q_weight=zeros(64), k_weight=zeros(64),
                                   q_out=zeros(3, 2, 64, dtype=b16), k_out=zeros(3, 1, 64, dtype=b16)),
            "attention": dict(q=zeros(3, 2, 64, dtype=b16), k=zeros(9, 1, 64, dtype=b16), v=zeros(9, 1, 64, dtype=b16), q_offsets=zeros(2, dtype=i32), k_begin=zeros(1, dtype=i32),
                              k_end=zeros(1, dtype=i32), scale=0.125, out=zeros(3, 2, 64, dtype=b16), lse=zeros(2, 3)),
        }


@pytest.fixture
def on_the_cpu(monkeypatch):
    """The checks take the CPU for the current device; what passes them is kept from the library."""
    monkeypatch.setattr(lop, "_current_device", lambda: -1)
    monkeypatch.setattr(lop, "_current_stream", lambda device: 0)

    class Library:
        def __init__(self):
            self.reached = []

        def __getattr__(self, name):
            def call(*args):
                self.reached.append(name)
                return 0
            return call
    library = Library()
    monkeypatch.setattr(lop, "_lib", library)
    return library


NAMES = list(Calls().of)


@pytest.mark.parametrize("name", NAMES)
def test_what_fits_reaches_the_library(name, on_the_cpu):
    getattr(lop, name)(**Calls().of[name])
    assert on_the_cpu.reached == ["lop_" + name]


PAIRS = [(name, key) for name, args in Calls().of.items() for key, t in args.items() if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("name,key", [(n, k) for n, k in PAIRS if Calls().of[n][k].is_floating_point()])
@pytest.mark.parametrize("recorded", [True, False])
def test_tensors_with_a_tangent_are_refused(name, key, recorded, on_the_cpu):
    """Forward-mode derivatives would be dropped; gradients need not be recorded for them."""
    args, fw = Calls().of[name], torch.autograd.forward_ad
    plain = dict(args)
    with torch.set_grad_enabled(recorded), fw.dual_level():
        getattr(lop, name)(**plain)                              # no tensor has one: as ever
        t = args[key]
        args[key] = fw.make_dual(t, t.clone())
        with pytest.raises(ValueError, match=f"{key}: .*tangent"):
            getattr(lop, name)(**args)
    assert on_the_cpu.reached == ["lop_" + name]
    getattr(lop, name)(**plain)


@pytest.mark.parametrize("name,key", [(n, k) for n, k in PAIRS if Calls().of[n][k].is_floating_point()])
def test_tensors_that_want_a_gradient_are_refused_while_it_is_recorded(name, key, on_the_cpu):
    args = Calls().of[name]
    args[key].requires_grad_()
    with pytest.raises(ValueError, match=f"{key}: .*gradient"):
        getattr(lop, name)(**args)
    assert not on_the_cpu.reached
    with torch.no_grad():
        getattr(lop, name)(**args)
    assert on_the_cpu.reached == ["lop_" + name]


@pytest.mark.parametrize("name,change", [
    ("quantize_blocks", lambda a: {k: t[:1].expand(1 << 31, -1) for k, t in a.items()}),
    ("rowwise_f8", lambda a: {k: t[:1].expand(1 << 31, -1) if k in ("x", "x_scale", "residual", "y") else t for k, t in a.items()}),
    ("head_norm_rope", lambda a: dict({k: t[:1].expand(1 << 31, -1, -1) if t.dim() == 3 else t for k, t in a.items()}, positions=None, freq=None)),
    ("head_norm_rope", lambda a: dict(a, eps="1")), ("attention", lambda a: dict(a, scale=None)),
    ("attention", lambda a: {k: t[:1].expand(1 << 31, -1, -1) if k in ("k", "v") else t for k, t in a.items()}),
    ("attention", lambda a: dict(a, max_keys=1 << 31)), ("attention", lambda a: dict(a, max_keys=-(1 << 40)))])
def test_numbers_that_the_library_does_not_hold_are_refused(name, change, on_the_cpu):
    with pytest.raises(ValueError):
        getattr(lop, name)(**change(Calls().of[name]))
    assert not on_the_cpu.reached


def test_a_workspace_is_asked_for_and_passed(on_the_cpu):
    args = Calls().of["attention"]
    lop.attention(**args, max_keys=lop.LOP_ATTENTION_CUT)
    lop.attention(**args, max_keys=1 << 20, workspace=torch.empty(64, dtype=torch.uint8))
    assert on_the_cpu.reached == ["lop_attention_workspace", "lop_attention", "lop_attention"]
