"""What heta_linear_xent, heta_adamw_multi and the calls on 8-bit whole numbers refuse, on the host, before any device call: the addresses here belong to
nothing.  Every case starts from arguments that would be launched and spoils one thing."""
import ctypes

import pytest
import torch

import paper_2408_09697_amd as heta
from paper_2408_09697_amd import binding as hb

BAD, SHAPE, UNSUPPORTED = hb.HETA_ERR_INVALID_ARG, hb.HETA_ERR_SHAPE, hb.HETA_ERR_UNSUPPORTED
F32, BF16, E4M3, I8 = hb.HETA_F32, hb.HETA_BF16, hb.HETA_E4M3, hb.HETA_I8
AT = {name: 0x10000000 * (i + 1) for i, name in enumerate("abcdefghijkl")}  # 256 MB apart
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    return hb.load_library()


@pytest.fixture(scope="module")
def handle():
    return ctypes.addressof(ctypes.create_string_buffer(4096))


def refused(lib, status, expect, needle=""):
    assert status == expect, (status, lib.heta_last_error())
    assert needle in lib.heta_last_error().decode()


XENT = dict(n_rows=100, d=64, n_classes=50, inp=AT["a"], ld_in=64, W=AT["b"], ld_w=50, bias=AT["c"], labels=AT["d"], loss=AT["e"], lse=AT["f"], mean=AT["g"], dt=F32)


@pytest.mark.parametrize("change,status,needle", [
    ({"n_rows": -1}, SHAPE, "n_rows"), ({"d": 0}, SHAPE, "width"), ({"n_classes": 0}, SHAPE, "classes"), ({"n_rows": 1 << 31}, UNSUPPORTED, "too many"),
    ({"n_classes": 2 ** 31 - 5, "ld_w": 2 ** 31}, UNSUPPORTED, "too many"), ({"dt": E4M3}, BAD, "dtype"), ({"dt": I8}, BAD, "dtype"), ({"inp": None}, BAD, "null in"),
    ({"W": None}, BAD, "null W"), ({"ld_in": 63}, SHAPE, "in"), ({"ld_w": 49}, SHAPE, "W"), ({"labels": None}, BAD, "labels"), ({"lse": None}, BAD, "lse"),
    ({"labels": AT["d"] + 4}, BAD, "aligned"), ({"inp": AT["a"] + 2}, BAD, "aligned"), ({"bias": AT["c"] + 2}, BAD, "aligned"), ({"mean": AT["g"] + 1}, BAD, "aligned"),
    ({"loss": AT["f"] + 40}, BAD, "overlap"), ({"mean": AT["e"] + 8}, BAD, "overlap"), ({"loss": AT["a"] + 400}, BAD, "overlap"), ({"lse": AT["d"]}, BAD, "overlap"),
    ({"mean": AT["b"] + 4}, BAD, "overlap"), ({"loss": AT["c"]}, BAD, "overlap")])
def test_loss(lib, handle, change, status, needle):
    refused(lib, lib.heta_linear_xent(handle, ctypes.byref(hb._XentArgs(**{**XENT, **change})), None), status, needle)


XENT_BWD = dict(n_rows=100, d=64, n_classes=50, inp=AT["a"], ld_in=64, W=AT["b"], ld_w=50, bias=AT["c"], labels=AT["d"], lse=AT["e"], grad_loss=AT["f"], mean=AT["g"], grad_in=AT["h"],
                ld_gi=64, dW=AT["i"], ld_dw=50, dbias=AT["j"], scale=1.0, dt=F32, dw_dt=F32)


@pytest.mark.parametrize("change,status,needle", [
    ({"n_rows": -1}, SHAPE, "n_rows"), ({"d": -1}, SHAPE, "width"), ({"n_classes": 0}, SHAPE, "classes"), ({"n_rows": 1 << 31}, UNSUPPORTED, "too many"), ({"dt": E4M3}, BAD, "dtype"),
    ({"dw_dt": I8}, BAD, "dtype"), ({"dw_dt": BF16}, UNSUPPORTED, "fp32"), ({"inp": None}, BAD, "null in"), ({"W": None}, BAD, "null W"), ({"ld_gi": 63}, SHAPE, "grad_in"),
    ({"ld_dw": 49}, SHAPE, "dW"), ({"labels": None}, BAD, "labels"), ({"lse": None}, BAD, "lse"), ({"labels": AT["d"] + 4}, BAD, "aligned"), ({"dbias": AT["j"] + 2}, BAD, "aligned"),
    ({"grad_loss": AT["f"] + 3}, BAD, "aligned"), ({"grad_in": AT["a"]}, BAD, "overlap"), ({"dW": AT["b"]}, BAD, "overlap"), ({"dbias": AT["c"]}, BAD, "overlap"),
    ({"dbias": AT["i"] + 400}, BAD, "overlap"), ({"grad_in": AT["e"]}, BAD, "overlap"), ({"dbias": AT["g"]}, BAD, "overlap"),
    ({"d": 1 << 17, "n_classes": 1 << 16, "ld_in": 1 << 17, "ld_gi": 1 << 17, "ld_w": 1 << 16, "ld_dw": 1 << 16, "n_rows": 4}, UNSUPPORTED, "elements")])
def test_gradients(lib, handle, change, status, needle):
    refused(lib, lib.heta_linear_xent_bwd(handle, ctypes.byref(hb._XentBwdArgs(**{**XENT_BWD, **change})), None), status, needle)


def test_null_handles_and_arguments(lib, handle):
    for call in (lib.heta_linear_xent, lib.heta_linear_xent_bwd):
        refused(lib, call(None, ctypes.byref(hb._XentArgs()), None), BAD, "null")
        refused(lib, call(handle, None, None), BAD, "null")


ADAMW = dict(W=AT["a"], ld_w=200, grad=AT["b"], ld_grad=200, m=AT["c"], v=AT["d"], ld_state=200, m_scale=None, v_scale=None, ld_scale=0, ids=AT["e"], n=60, rows=100, d=200, dt=BF16,
             grad_dt=F32, state_dt=F32, weight_decay=0.1, seed=1)
ADAMW8 = dict(ADAMW, state_dt=E4M3, m_scale=AT["f"], v_scale=AT["g"], ld_scale=2)
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)


def adamw(lib, items, **change):
    arr = (hb._AdamwItem * max(1, len(items)))(*[hb._AdamwItem(**it) for it in items])
    h = {**HYPER, **change}
    return lib.heta_adamw_multi(len(items), ctypes.cast(arr, ctypes.c_void_p), h["lr"], h["beta1"], h["beta2"], h["eps"], h["step"], None)


@pytest.mark.parametrize("base,change,status,needle", [
    (ADAMW, {"W": None}, BAD, "null W"), (ADAMW, {"grad": None}, BAD, "null grad"), (ADAMW, {"m": None}, BAD, "null m"), (ADAMW, {"v": None}, BAD, "null v"),
    (ADAMW, {"d": 0}, SHAPE, "d > 0"), (ADAMW, {"n": -1}, SHAPE, "counts"), (ADAMW, {"rows": -1}, SHAPE, "counts"), (ADAMW, {"dt": E4M3}, BAD, "dtype"), (ADAMW, {"grad_dt": 7}, BAD, "dtype"),
    (ADAMW, {"state_dt": BF16}, BAD, "dtype"), (ADAMW, {"state_dt": I8}, BAD, "dtype"), (ADAMW, {"ld_w": 199}, SHAPE, "W"), (ADAMW, {"ld_grad": 1}, SHAPE, "grad"), (ADAMW, {"ld_state": 199}, SHAPE, "m"),
    (ADAMW8, {"ld_scale": 1}, SHAPE, "m_scale"), (ADAMW, {"m_scale": AT["f"]}, BAD, "scales"), (ADAMW8, {"v_scale": None}, BAD, "scales"), (ADAMW, {"ids": None, "n": 101}, SHAPE, "gradient rows"),
    (ADAMW, {"ids": AT["e"] + 4}, BAD, "aligned"), (ADAMW, {"W": AT["a"] + 1}, BAD, "aligned"), (ADAMW, {"m": AT["c"] + 2}, BAD, "aligned"), (ADAMW8, {"m_scale": AT["f"] + 2}, BAD, "aligned"),
    (ADAMW, {"weight_decay": -1.0}, BAD, "weight_decay"), (ADAMW, {"weight_decay": NAN}, BAD, "weight_decay"), (ADAMW, {"m": AT["a"]}, BAD, "overlaps"), (ADAMW, {"v": AT["c"] + 400}, BAD, "overlaps"),
    (ADAMW, {"grad": AT["a"] + 400}, BAD, "overlaps"), (ADAMW, {"ids": AT["c"] + 8}, BAD, "overlaps"), (ADAMW8, {"v_scale": AT["f"] + 4}, BAD, "overlaps"), (ADAMW8, {"m_scale": AT["c"]}, BAD, "overlaps"),
    (ADAMW, {"d": 2 ** 31 - 100, "ld_w": 2 ** 31, "ld_grad": 2 ** 31, "ld_state": 2 ** 31}, UNSUPPORTED, "too wide")])
def test_update(lib, base, change, status, needle):
    refused(lib, adamw(lib, [{**base, **change}]), status, needle)
    # an item that would be launched in front of it is not
    far = {**ADAMW, **{k: ADAMW[k] + 0x700000000 for k in ("W", "grad", "m", "v", "ids")}}
    refused(lib, adamw(lib, [far, {**base, **change}]), status, needle)


def test_update_of_arrays_that_two_items_share(lib):
    far = {k: ADAMW[k] + 0x700000000 for k in ("W", "grad", "m", "v", "ids")}
    for name in ("W", "m", "v"):
        refused(lib, adamw(lib, [ADAMW, {**ADAMW, **far, name: ADAMW["W"] + 4000}]), BAD, "overlaps")
    refused(lib, adamw(lib, [ADAMW, {**ADAMW, **far, "grad": ADAMW["v"]}]), BAD, "overlaps")
    refused(lib, adamw(lib, [ADAMW, ADAMW]), BAD, "overlaps")


@pytest.mark.parametrize("change,needle", [({"step": 0}, "step"), ({"beta1": 1.0}, "beta"), ({"beta2": -0.1}, "beta"), ({"beta2": NAN}, "beta"), ({"eps": -1.0}, "eps"), ({"eps": NAN}, "eps")])
def test_hyper_parameters(lib, change, needle):
    refused(lib, adamw(lib, [ADAMW], **change), BAD, needle)
    refused(lib, lib.heta_adamw_multi(-1, None, 1e-3, 0.9, 0.999, 1e-8, 1, None), BAD, "list")
    refused(lib, lib.heta_adamw_multi(1, None, 1e-3, 0.9, 0.999, 1e-8, 1, None), BAD, "list")


I8_LINEAR = dict(n_rows=100, d_in=64, d_out=48, inp=AT["a"], ld_in=64, W=AT["b"], ld_w=64, bias=AT["c"], out=AT["f"], ld_out=48, in_dt=I8, w_dt=I8, out_dt=F32, act=0, in_scale=AT["g"],
                 w_scale=AT["h"])


@pytest.mark.parametrize("change,status,needle", [
    ({"coarse_sums": 1}, BAD, "coarse"), ({"w_dt": E4M3}, UNSUPPORTED, "one type"), ({"out_dt": I8}, BAD, "outputs"), ({"in_scale": None}, BAD, "scales"), ({"w_scale": None}, BAD, "scales"),
    ({"ld_w": 63}, SHAPE, "W"), ({"d_in": 1 << 17, "ld_in": 1 << 17, "ld_w": 1 << 17}, UNSUPPORTED, "2^17"), ({"out": AT["a"] + 16}, BAD, "overlaps"), ({"out": AT["g"]}, BAD, "overlaps")])
def test_products_of_whole_numbers(lib, handle, change, status, needle):
    refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**{**I8_LINEAR, **change})), None), status, needle)


ROWS = dict(n=100, d=64, x=AT["a"], x_dt=F32, ld_x=64, out=AT["b"], ld_out=64, scale=AT["c"], stream=None)


@pytest.mark.parametrize("change,status,needle", [
    ({"n": -1}, SHAPE, "n_rows"), ({"d": 0}, SHAPE, "d > 0"), ({"d": 2 ** 31 - 5}, UNSUPPORTED, "wide"), ({"x_dt": I8}, BAD, "dtype"), ({"x": None}, BAD, "null x"), ({"out": None}, BAD, "null out"),
    ({"scale": None}, BAD, "scale"), ({"ld_x": 63}, SHAPE, "x"), ({"ld_out": 63}, SHAPE, "out"), ({"x": AT["a"] + 2}, BAD, "aligned"), ({"scale": AT["c"] + 2}, BAD, "scale"),
    ({"out": AT["a"]}, BAD, "overlaps"), ({"scale": AT["a"]}, BAD, "overlaps"), ({"scale": AT["b"] + 64}, BAD, "overlaps")])
def test_rows_of_whole_numbers(lib, change, status, needle):
    refused(lib, lib.heta_linear_rows_i8(*{**ROWS, **change}.values()), status, needle)


PACK = dict(W=AT["a"], w_dt=F32, ld_w=48, d_in=64, d_out=48, packed=AT["b"], ld_packed=64, scale=AT["c"], stream=None)


@pytest.mark.parametrize("change,status,needle", [
    ({"w_dt": I8}, BAD, "dtype"), ({"d_in": 0}, SHAPE, "widths"), ({"W": None}, BAD, "null W"), ({"packed": None}, BAD, "null packed"), ({"scale": None}, BAD, "scale"), ({"ld_w": 47}, SHAPE, "W"),
    ({"ld_packed": 63}, SHAPE, "packed"), ({"packed": AT["a"]}, BAD, "overlaps"), ({"scale": AT["b"]}, BAD, "overlaps")])
def test_weights_of_whole_numbers(lib, change, status, needle):
    refused(lib, lib.heta_linear_pack_i8(*{**PACK, **change}.values()), status, needle)


def test_tensors_of_the_wrong_kind():
    """What the binding refuses of tensors: they have to be on the device in the first place."""
    W, g = torch.zeros(4, 8), torch.zeros(4, 8)
    with pytest.raises((heta.HetaError, TypeError, ValueError)):
        heta.heta_adamw_plan([(W, (W.clone(), W.clone()), g)])
    with pytest.raises(ValueError):
        heta.heta_adamw_state(W, 16)
    state = heta.heta_adamw_state(torch.zeros(5, 300), 8)
    assert [tuple(x.shape) for x in state] == [(5, 300), (5, 3), (5, 300), (5, 3)]
    assert [tuple(x.shape) for x in heta.heta_adamw_state(torch.zeros(7))] == [(7,), (7,)]
