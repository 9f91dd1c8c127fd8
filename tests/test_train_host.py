"""Host-side checks of the training step's calls that need no GPU: the
library exports what cerar_train.h declares, the ctypes mirrors have its
layout, bad arguments are refused before the device is touched, and the
oracle's formats agree with the formats' definition and with torch's casts."""

import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from conftest import ROOT
from oracle import train as O
from paper_2609_23898_amd import cerar as C
from paper_2609_23898_amd import train as T

HEADER = os.path.join(ROOT, "include", "cerar_train.h")
FP8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def _text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_library_exports_every_declared_function():
    names = sorted(set(re.findall(r"\b(cerar_[a-z0-9_]+)\s*\(", _text())))
    assert names == sorted(T.SIGNATURES) and len(names) == 9
    for n in names:
        assert hasattr(T.lib(), n), n


@pytest.mark.parametrize("name,mirror", [("cerar_tensor", T.TensorDesc), ("cerar_adamw", T.AdamWDesc),
                                         ("cerar_adamw_values", T.AdamWValues), ("cerar_blocks", T.BlocksDesc)])
def test_struct_layouts_match_header(name, mirror):
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", _text()).group(1)
    fields = re.findall(r"([A-Za-z_][A-Za-z0-9_]*)\s*(?=[,;])", body)
    assert fields == [f for f, _ in mirror._fields_]


# --- the oracle's formats -----------------------------------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_code_values_match_torch(fmt):
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(O.code_values(fmt), codes.view(FP8[fmt]).double().numpy())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_nearest_matches_torch_cast(fmt):
    rng = np.random.default_rng(1)
    x = (rng.standard_normal(20000) * 2.0 ** rng.uniform(-20, 12, 20000)).clip(-O.TOP[fmt], O.TOP[fmt])
    t = O.positive(fmt)
    x = np.concatenate([x, t, (t[1:] + t[:-1]) / 2, [0.0, -0.0]]).astype(np.float32)
    np.testing.assert_array_equal(O.nearest(x.astype(np.float64), fmt),
                                  torch.from_numpy(x).to(FP8[fmt]).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_scale_exponent_is_the_least_that_fits(fmt):
    a = np.concatenate([[0.0, O.TOP[fmt], np.nextafter(O.TOP[fmt], 1e9), 2.0 ** -149, 3.4e38],
                        2.0 ** np.random.default_rng(2).uniform(-100, 100, 200)])
    k = O.scale_exponent(a, fmt)
    assert (a <= O.TOP[fmt] * 2.0 ** k.astype(float)).all()
    assert ((k == -127) | (a > O.TOP[fmt] * 2.0 ** (k - 1.0))).all()


def test_rounding_by_chance_is_unbiased_and_keeps_codes():
    for fmt in ("e4m3", "e5m2"):
        t = O.positive(fmt)
        exact = t[1:].copy()
        codes, k = O.round_by_chance(np.concatenate([exact, [t[-1]]]), fmt, np.full(len(exact) + 1, 65535.0))
        assert (codes[:-1] == np.arange(1, len(t))).all() and (k == 0).all()
        x = np.array([O.TOP[fmt], 0.37 * O.TOP[fmt], 1.3 * t[1]])
        got = np.array([O.code_values(fmt)[O.round_by_chance(x, fmt, np.full(3, float(r)))[0]] for r in range(0, 65536, 64)])
        np.testing.assert_allclose(got.mean(0), x, rtol=2e-3)


# --- refusals ------------------------------------------------------------------------

def _tensor(**kw):
    base = 1 << 20
    d = dict(n=100, grad=base, param=base * 2, m=base * 3, v=base * 4, grad_type=0, param_type=0, lr_scale=1.0,
             weight_decay=0.0)
    d.update(kw)
    return T.TensorDesc(**d)


@pytest.mark.parametrize("bits,change,text", [
    (16, {}, "state_bits"), (32, {"grad": None}, "grad is NULL"), (32, {"m": None}, "m is NULL"),
    (8, {}, "m_scale is NULL"), (32, {"param": (1 << 21) + 2}, "not aligned"),
    (32, {"grad": (1 << 20) + 1, "grad_type": 1}, "not aligned"), (32, {"grad_type": 2}, "unknown type"),
    (32, {"m": (1 << 21) + 16}, "overlap"), (32, {"copy": (1 << 20) + 8}, "overlap"),
    (32, {"grad": (1 << 21)}, "overlap"), (32, {"lr_scale": math.nan}, "not finite"),
    (32, {"weight_decay": math.inf}, "not finite"), (32, {"n": (1 << 40) + 1}, "2\\^40"),
    (32, {"m_scale": 1 << 24}, "without 8-bit states")])
def test_set_refuses(bits, change, text):
    h = ctypes.c_void_p()
    with pytest.raises(C.CerarError, match=text) as e:
        C._check(T.lib().cerar_tensors_create(1, ctypes.byref(_tensor(**change)), bits, ctypes.byref(h)))
    assert e.value.status == -1 and not h


def test_set_refuses_tensors_that_overlap_each_other():
    base = 1 << 20
    two = (T.TensorDesc * 2)(_tensor(), _tensor(grad=base * 5, param=base * 6, m=base * 7, v=base * 4 + 399))
    h = ctypes.c_void_p()
    assert T.lib().cerar_tensors_create(2, two, 32, ctypes.byref(h)) == -1
    two[1].v = base * 4 + 396
    assert T.lib().cerar_tensors_create(2, two, 32, ctypes.byref(h)) == -1
    assert T.lib().cerar_tensors_create(0, two, 32, ctypes.byref(h)) == -1
    assert T.lib().cerar_tensors_create(2, None, 32, ctypes.byref(h)) == -1


@pytest.mark.parametrize("change", [{"step": 0}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": math.nan},
                                    {"eps": 0.0}, {"eps": math.inf}, {"lr": math.nan}, {"grad_scale": math.inf}])
def test_step_settings_refused(change):
    with pytest.raises(C.CerarError) as e:
        T.adamw_values(**{"step": 1, "lr": 1e-3, **change})
    assert e.value.status == -1


@pytest.mark.parametrize("change", [{"eps": 1e-39}, {"eps": 1e-60}, {"eps": 1e39}, {"lr": 1e39}, {"grad_scale": -1e39},
                                    {"lr": 1e30, "beta1": 1 - 2.0 ** -40}])
def test_step_settings_beyond_fp32_are_refused(change):
    with pytest.raises(C.CerarError) as e:
        T.adamw_values(**{"step": 1, "lr": 1e-3, **change})
    assert e.value.status == -1
    T.adamw_values(1, 1e-3, eps=2.0 ** -126)


def test_negative_steps_are_refused():
    """A negative number would wrap to one of some 2^64, whose bias corrections are 1."""
    for step in (-1, -(1 << 63)):
        with pytest.raises(ValueError, match="first step is 1"):
            T.adamw_values(step, 1e-3)
        with pytest.raises(ValueError, match="first step is 1"):
            T.adamw_step(None, step, 1e-3)


def test_step_values():
    v = T.AdamWValues.from_buffer_copy(bytes(T.adamw_values(3, 1e-2, 0.8, 0.99, 1e-6, 0.25, 5).numpy()))
    f = np.float32
    assert (v.beta1, v.rest1, v.beta2, v.rest2) == (0.8, 1 - 0.8, 0.99, 1 - 0.99)
    assert (v.lr, v.eps, v.grad_scale) == tuple(map(f, (1e-2, 1e-6, 0.25)))
    assert v.step_size == f(1e-2 / (1 - 0.8 ** 3)) and v.root2 == f(1 / math.sqrt(1 - 0.99 ** 3))
    assert v.key == O.mixed(5 + 4 * O.GOLDEN & O.MASK)


def _blocks(rows, cols, codes=1 << 30, scales=1 << 40, fmt=0):
    return T.BlocksDesc(codes, scales, rows, cols, fmt)


def test_quantize_refuses():
    q = T.lib().cerar_quantize_blocks
    x, ok_r = 1 << 20, _blocks(10, 200)
    r = ctypes.byref(ok_r)
    for args, text in [
            ((x, 0, 10, 200, 200, 0, None, None), b"no destination"), ((x, 2, 10, 200, 200, 0, r, None), b"unknown type"),
            ((x, 0, 10, 200, 199, 0, r, None), b"below cols"), ((None, 0, 10, 200, 200, 0, r, None), b"NULL x"),
            ((x + 2, 0, 10, 200, 200, 0, r, None), b"not aligned"), ((x, 0, 10, 201, 201, 0, r, None), b"by_row is"),
            ((x, 0, 10, 200, 200, 0, r, r), b"by_col is"), ((1 << 30, 0, 10, 200, 200, 0, r, None), b"overlap"),
            ((x, 0, 10, 200, 200, 0, ctypes.byref(_blocks(10, 200, (1 << 30) + 8)), None), b"16-byte"),
            ((x, 0, 10, 200, 200, 0, ctypes.byref(_blocks(10, 200, None)), None), b"NULL buffer"),
            ((x, 0, 10, 200, 200, 0, ctypes.byref(_blocks(10, 200, fmt=2)), None), b"unknown format"),
            ((x, 0, 10, 200, 200, 0, r, ctypes.byref(_blocks(200, 10, 1 << 31, 1 << 41, 1))), b"different formats"),
            ((x, 0, 10, 200, 200, 0, r, ctypes.byref(_blocks(200, 10, 1 << 30, 1 << 41))), b"overlap"),
            ((x, 0, 1 << 31, 200, 200, 0, r, None), b"2^31")]:
        assert q(*args, None) == -1 and text in T.lib().cerar_last_error(), (text, T.lib().cerar_last_error())
    assert q(None, 0, 0, 200, 200, 0, ctypes.byref(_blocks(0, 200, None, None)), None, None) == 0


def test_products_refuse():
    mm, lin = T.lib().cerar_matmul_blocks, T.lib().cerar_linear_blocks
    a, b, out, ws = _blocks(10, 200), _blocks(30, 200, 1 << 31, 1 << 41), 1 << 33, 1 << 42
    pa, pb = ctypes.byref(a), ctypes.byref(b)
    other = ctypes.byref(_blocks(30, 201, 1 << 31, 1 << 41))
    for args, text in [((None, pb, out, 0, 30, 0, ws), b"NULL"), ((pa, other, out, 0, 30, 0, ws), b"200 columns"),
                       ((pa, pb, None, 0, 30, 0, ws), b"NULL out"), ((pa, pb, out, 0, 29, 0, ws), b"below N"),
                       ((pa, pb, out + 2, 0, 30, 0, ws), b"not aligned"), ((pa, pb, out, 1, 30, 1, ws), b"accumulate"),
                       ((pa, pb, out, 3, 30, 0, ws), b"unknown out_type"), ((pa, pb, 1 << 31, 0, 30, 0, ws), b"overlap"),
                       ((pa, pb, (1 << 40) - 400, 0, 30, 0, ws), b"overlap")]:
        args = args[:6] + (0,) + args[6:]
        assert mm(*args, None) == -1 and text in T.lib().cerar_last_error(), (text, T.lib().cerar_last_error())
    x = 1 << 20
    for args, text in [((x, 0, 10, 200, None, out, 0, 30, ws), b"NULL"), ((x, 5, 10, 200, pb, out, 0, 30, ws), b"unknown type"),
                       ((x, 0, 10, 199, pb, out, 0, 30, ws), b"below cols"), ((None, 0, 10, 200, pb, out, 0, 30, ws), b"NULL x"),
                       ((x, 0, 10, 200, pb, x + 40, 0, 30, ws), b"overlap"), ((x, 0, 10, 200, pb, out, 0, 30, None), b"NULL ws"),
                       ((x, 0, 10, 200, pb, out, 0, 30, ws + 4), b"16-byte"), ((x, 0, 10, 200, pb, out, 0, 30, out), b"overlap"),
                       ((x + 1, 1, 10, 200, pb, out, 0, 30, ws), b"not aligned")]:
        args = args[:8] + (0,) + args[8:]
        assert lin(*args, None) == -1 and text in T.lib().cerar_last_error(), (text, T.lib().cerar_last_error())
    assert mm(pa, pb, out, 0, 30, 0, 2, ws, None) == -1 and b"unknown sums" in T.lib().cerar_last_error()
    with pytest.raises(C.CerarError):
        T.matmul_workspace_bytes(1 << 31, 1, 1)


def test_more_work_than_a_launch_takes_is_refused():
    out, ws = 1 << 60, 1 << 61
    a, b = _blocks(1, 2048), _blocks(1 << 30, 2048, 1 << 50, 1 << 55)
    assert T.lib().cerar_matmul_blocks(ctypes.byref(a), ctypes.byref(b), out, 0, 1 << 30, 0, 0, ws, None) == -1
    assert b"too large" in T.lib().cerar_last_error()
    a = _blocks(1 << 20, 128)
    b = _blocks(1 << 30, 128, 1 << 50, 1 << 55)
    assert T.lib().cerar_matmul_blocks(ctypes.byref(a), ctypes.byref(b), out, 0, 1 << 30, 0, 0, ws, None) == -1
    assert b"too large" in T.lib().cerar_last_error()
    big = _blocks((1 << 31) - 1, 4096, 1 << 50, 1 << 55)
    assert T.lib().cerar_quantize_blocks(1 << 20, 1, (1 << 31) - 1, 4096, 4096, 1, ctypes.byref(big), None, None) == -1
    assert b"too large" in T.lib().cerar_last_error()


@pytest.mark.parametrize("ld", [1 << 54, 1 << 61, (1 << 62) + 50, (1 << 63) + 200, (1 << 64) - 1])
def test_row_strides_beyond_the_address_space_are_refused(ld):
    """Their byte ranges wrap around: without a check of their own they pass the one for overlaps."""
    a, b, out, ws = _blocks(10, 200), _blocks(30, 200, 1 << 31, 1 << 41), 1 << 33, 1 << 42
    pa, pb = ctypes.byref(a), ctypes.byref(b)
    for status in (T.lib().cerar_quantize_blocks(1 << 20, 0, 10, 200, ld, 0, pa, None, None),
                   T.lib().cerar_quantize_blocks(1 << 20, 1, 10, 200, ld, 1, pa, None, None),
                   T.lib().cerar_matmul_blocks(pa, pb, out, 0, ld, 0, 0, ws, None),
                   T.lib().cerar_linear_blocks(1 << 20, 1, 10, ld, pb, out, 0, 30, 0, ws, None),
                   T.lib().cerar_linear_blocks(1 << 20, 1, 10, 200, pb, out, 1, ld, 0, ws, None)):
        assert status == -1 and b"address space" in T.lib().cerar_last_error()


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 4)
    for call in (lambda: T.GradSet([x]), lambda: T.TensorSet([x], [x]), lambda: T.quantize_blocks(x, rows=object()),
                 lambda: T.Blocks(torch.zeros((4, 128), dtype=torch.float8_e4m3fn), torch.zeros((1, 4, 4), dtype=torch.uint8), 4)):
        with pytest.raises(ValueError, match="must be a tensor on the GPU"):
            call()
    with pytest.raises(ValueError, match="must be a Blocks"):
        T.matmul_blocks(x, x, x)
    with pytest.raises(ValueError, match="state_bits"):
        T.TensorSet([x], [x], state_bits=16)
    with pytest.raises(ValueError, match="rows or cols"):
        T.quantize_blocks(x)
    with pytest.raises(ValueError, match="1 params, 0 grads"):
        T.TensorSet([x], [])
