"""What heta_rms_norm, heta_linear and heta_muon_multi (and their backward calls) refuse, on the host, before any device call: the
addresses here belong to nothing.  Every case starts from arguments that would be launched and spoils one thing."""
import ctypes

import pytest

from paper_2408_09697_amd import binding as hb

BAD, SHAPE, UNSUPPORTED = hb.HETA_ERR_INVALID_ARG, hb.HETA_ERR_SHAPE, hb.HETA_ERR_UNSUPPORTED
F32, BF16, E4M3 = hb.HETA_F32, hb.HETA_BF16, hb.HETA_E4M3
AT = {name: 0x10000000 * (i + 1) for i, name in enumerate("abcdefghijkl")}  # 256 MB apart


@pytest.fixture(scope="module")
def lib():
    return hb.load_library()


@pytest.fixture(scope="module")
def handle():
    return ctypes.addressof(ctypes.create_string_buffer(4096))


def refused(lib, status, expect, needle=""):
    assert status == expect, (status, lib.heta_last_error())
    assert needle in lib.heta_last_error().decode()


NORM = dict(n=100, d=64, x=AT["a"], x_dt=F32, ld_x=64, res=AT["b"], ld_res=64, gamma=AT["c"], eps=1e-6, sum=AT["d"], ld_sum=64, out=AT["e"], out_dt=F32, ld_out=64,
            scale=None, rstd=AT["f"], stream=None)


@pytest.mark.parametrize("change,status,needle", [
    ({"n": -1}, SHAPE, "n_rows"), ({"d": 0}, SHAPE, "d > 0"), ({"x_dt": 7}, BAD, "dtype"), ({"out_dt": 9}, BAD, "dtype"), ({"x_dt": E4M3}, BAD, "dtype"),
    ({"eps": -1.0}, BAD, "eps"), ({"eps": float("nan")}, BAD, "eps"), ({"x": None}, BAD, "null x"), ({"out": None}, BAD, "null out"), ({"ld_x": 63}, SHAPE, "x"),
    ({"ld_out": 10}, SHAPE, "out"), ({"ld_res": 0}, SHAPE, "residual"), ({"ld_sum": 63}, SHAPE, "sum"), ({"out_dt": E4M3}, BAD, "scales"), ({"scale": AT["g"]}, BAD, "scales"),
    ({"x": AT["a"] + 2}, BAD, "aligned"), ({"gamma": AT["c"] + 1}, BAD, "aligned"), ({"x_dt": BF16}, UNSUPPORTED, "bf16"), ({"out": AT["a"]}, BAD, "overlaps"),
    ({"sum": AT["a"] + 256}, BAD, "overlaps"), ({"out": AT["d"]}, BAD, "overlaps"), ({"sum": AT["b"], "ld_sum": 128}, BAD, "overlaps")])
def test_norm(lib, change, status, needle):
    refused(lib, lib.heta_rms_norm(*{**NORM, **change}.values()), status, needle)


NORM_BWD = dict(g=1, n=100, d=64, x=AT["a"], x_dt=F32, ld_x=64, gamma=AT["c"], rstd=AT["d"], go=AT["e"], go_dt=F32, ld_go=64, gs=AT["f"], ld_gs=64, gx=AT["g"], ld_gx=64,
                gg=AT["h"], stream=None)


@pytest.mark.parametrize("change,status,needle", [
    ({"g": None}, BAD, "handle"), ({"n": -1}, SHAPE, "n_rows"), ({"d": 0}, SHAPE, "d > 0"), ({"x_dt": 3}, BAD, "dtype"), ({"go_dt": E4M3}, BAD, "dtype"),
    ({"x_dt": BF16}, UNSUPPORTED, "bf16"), ({"rstd": None}, BAD, "rstd"), ({"x": None}, BAD, "null x"), ({"go": None}, BAD, "grad_out"), ({"gx": None}, BAD, "grad_x"),
    ({"ld_go": 1}, SHAPE, "grad_out"), ({"gx": AT["a"]}, BAD, "overlaps"), ({"gx": AT["e"]}, BAD, "overlaps"), ({"gx": AT["f"], "ld_gx": 65}, BAD, "overlaps"),
    ({"gg": AT["h"] + 2}, BAD, "aligned")])
def test_norm_backward(lib, handle, change, status, needle):
    a = {**NORM_BWD, **change}
    a["g"] = handle if a["g"] else None
    refused(lib, lib.heta_rms_norm_bwd(*a.values()), status, needle)


LINEAR = dict(n_rows=100, d_in=64, d_out=48, inp=AT["a"], ld_in=64, W=AT["b"], ld_w=48, bias=AT["c"], residual=AT["d"], ld_res=48, pre=AT["e"], ld_pre=48, out=AT["f"], ld_out=48,
              in_dt=F32, w_dt=F32, out_dt=F32, act=hb.HETA_ACT_GELU)
LINEAR8 = dict(LINEAR, in_dt=E4M3, w_dt=E4M3, ld_w=64, in_scale=AT["g"], w_scale=AT["h"])


@pytest.mark.parametrize("base,change,status,needle", [
    (LINEAR, {"n_rows": -1}, SHAPE, "n_rows"), (LINEAR, {"d_in": 0}, SHAPE, "widths"), (LINEAR, {"d_out": -4}, SHAPE, "widths"), (LINEAR, {"act": 4}, BAD, "act"),
    (LINEAR, {"act": -1}, BAD, "act"), (LINEAR, {"in_dt": 5}, BAD, "dtype"), (LINEAR, {"out_dt": E4M3}, BAD, "outputs"), (LINEAR, {"w_dt": BF16}, UNSUPPORTED, "one type"),
    (LINEAR, {"out_dt": BF16}, UNSUPPORTED, "fp32"), (LINEAR, {"in_scale": AT["g"]}, BAD, "scales"), (LINEAR8, {"w_scale": None}, BAD, "scales"),
    (LINEAR8, {"in_scale": None}, BAD, "scales"), (LINEAR, {"coarse_sums": 1}, BAD, "coarse"), (LINEAR, {"inp": None}, BAD, "null in"), (LINEAR, {"W": None}, BAD, "null W"),
    (LINEAR, {"out": None}, BAD, "null out"), (LINEAR, {"ld_in": 63}, SHAPE, "in"), (LINEAR, {"ld_w": 47}, SHAPE, "W"), (LINEAR8, {"ld_w": 63}, SHAPE, "W"),
    (LINEAR, {"ld_out": 47}, SHAPE, "out"), (LINEAR, {"ld_res": 1}, SHAPE, "residual"), (LINEAR, {"ld_pre": 1}, SHAPE, "pre"), (LINEAR, {"inp": AT["a"] + 2}, BAD, "aligned"),
    (LINEAR, {"bias": AT["c"] + 2}, BAD, "aligned"), (LINEAR, {"out": AT["a"]}, BAD, "overlaps"), (LINEAR, {"out": AT["b"] + 16}, BAD, "overlaps"),
    (LINEAR, {"pre": AT["f"]}, BAD, "overlaps"), (LINEAR, {"pre": AT["d"]}, BAD, "overlaps"), (LINEAR, {"out": AT["d"], "ld_out": 64}, BAD, "overlaps")])
def test_linear(lib, handle, base, change, status, needle):
    refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**{**base, **change})), None), status, needle)


LINEAR_BWD = dict(n_rows=100, d_in=64, d_out=48, dt=F32, dw_dt=F32, act=hb.HETA_ACT_SILU, in_act=hb.HETA_ACT_RELU, inp=AT["a"], ld_inp=64, W=AT["b"], ld_W=48, grad_out=AT["c"], ld_grad_out=48,
                  pre=AT["d"], ld_pre=48, grad_pre=AT["e"], ld_grad_pre=48, grad_in=AT["f"], ld_grad_in=64, in_pre=AT["g"], ld_in_pre=64, dW=AT["h"], ld_dW=48, dbias=AT["i"])


@pytest.mark.parametrize("change,status,needle", [
    ({"n_rows": -1}, SHAPE, "n_rows"), ({"d_in": 0}, SHAPE, "widths"), ({"act": 9}, BAD, "act"), ({"in_act": 9}, BAD, "act"), ({"dt": E4M3}, BAD, "dtype"), ({"dw_dt": 8}, BAD, "dtype"),
    ({"dw_dt": BF16}, UNSUPPORTED, "fp32"), ({"grad_out": None}, BAD, "grad_out"), ({"pre": None}, BAD, "pre"), ({"grad_pre": None}, BAD, "grad_pre"), ({"W": None}, BAD, "W"),
    ({"in_pre": None}, BAD, "in_pre"), ({"inp": None}, BAD, "null in"), ({"ld_dW": 47}, SHAPE, "dW"), ({"ld_grad_in": 63}, SHAPE, "grad_in"), ({"ld_W": 1}, SHAPE, "W"),
    ({"dbias": AT["i"] + 1}, BAD, "aligned"), ({"grad_in": AT["a"]}, BAD, "overlaps"), ({"grad_in": AT["e"]}, BAD, "overlap"), ({"dW": AT["b"]}, BAD, "overlaps"),
    ({"grad_pre": AT["c"] + 192}, BAD, "overlaps"), ({"dbias": AT["h"]}, BAD, "overlap")])
def test_linear_backward(lib, handle, change, status, needle):
    refused(lib, lib.heta_linear_bwd(handle, ctypes.byref(hb._LinearBwdArgs(**{**LINEAR_BWD, **change})), None), status, needle)
    refused(lib, lib.heta_linear_bwd(None, ctypes.byref(hb._LinearBwdArgs(**LINEAR_BWD)), None), BAD, "null")


PACK = dict(W=AT["a"], dt=F32, ld=48, d_in=64, d_out=48, packed=AT["b"], ld_p=64, scale=AT["c"], stream=None)


@pytest.mark.parametrize("change,status,needle", [
    ({"dt": E4M3}, BAD, "dtype"), ({"d_in": 0}, SHAPE, "widths"), ({"ld": 47}, SHAPE, "W"), ({"ld_p": 63}, SHAPE, "packed"), ({"W": None}, BAD, "W"), ({"packed": None}, BAD, "packed"),
    ({"scale": None}, BAD, "scale"), ({"packed": AT["a"] + 64}, BAD, "overlaps"), ({"scale": AT["b"]}, BAD, "overlaps")])
def test_pack(lib, change, status, needle):
    refused(lib, lib.heta_linear_pack_e4m3(*{**PACK, **change}.values()), status, needle)


ITEM = dict(W=AT["a"], ld_w=48, m=AT["b"], ld_m=48, grad=AT["c"], ld_grad=48, rows=64, cols=48, dt=F32, grad_dt=F32)
SECOND = dict(ITEM, W=AT["d"], m=AT["e"], grad=AT["f"])
HYPER = dict(lr=0.02, momentum=0.9, nesterov=1, wd=0.0, eps=1e-7, steps=5)


@pytest.mark.parametrize("change,hyper,status,needle", [
    ({"rows": 0}, {}, SHAPE, "item 1"), ({"cols": -1}, {}, SHAPE, "item 1"), ({"ld_w": 47}, {}, SHAPE, "item 1"), ({"ld_m": 1}, {}, SHAPE, "item 1"), ({"ld_grad": 0}, {}, SHAPE, "item 1"),
    ({"W": None}, {}, BAD, "null"), ({"m": None}, {}, BAD, "null"), ({"grad": None}, {}, BAD, "null"), ({"dt": E4M3}, {}, BAD, "dtype"), ({"grad_dt": 5}, {}, BAD, "dtype"),
    ({"m": AT["e"] + 2}, {}, BAD, "aligned"), ({"grad": AT["d"]}, {}, BAD, "overlaps"), ({"W": AT["a"] + 64}, {}, BAD, "overlaps"), ({"grad": AT["b"]}, {}, BAD, "overlaps"),
    ({"rows": 1 << 20, "cols": 1 << 20, "ld_w": 1 << 20, "ld_m": 1 << 20, "ld_grad": 1 << 20}, {}, UNSUPPORTED, "large"),
    ({}, {"momentum": 1.0}, BAD, "momentum"), ({}, {"momentum": -0.1}, BAD, "momentum"), ({}, {"eps": 0.0}, BAD, "eps"), ({}, {"steps": -1}, BAD, "steps"), ({}, {"steps": 65}, BAD, "steps"),
    ({}, {"wd": -1.0}, BAD, "weight_decay"), ({}, {"lr": float("inf")}, BAD, "lr"), ({}, {"lr": float("nan")}, BAD, "lr")])
def test_muon(lib, handle, change, hyper, status, needle):
    items = (hb._MuonItem * 2)(hb._MuonItem(**ITEM), hb._MuonItem(**{**SECOND, **change}))
    refused(lib, lib.heta_muon_multi(handle, 2, ctypes.byref(items), *{**HYPER, **hyper}.values(), None), status, needle)


def test_muon_lists(lib, handle):
    refused(lib, lib.heta_muon_multi(None, 0, None, *HYPER.values(), None), BAD, "handle")
    refused(lib, lib.heta_muon_multi(handle, 1, None, *HYPER.values(), None), BAD, "list")
    refused(lib, lib.heta_muon_multi(handle, -1, None, *HYPER.values(), None), BAD, "list")
    assert lib.heta_muon_multi(handle, 0, None, *HYPER.values(), None) == hb.HETA_OK


def test_other_calls_do_not_know_the_new_types(lib):
    refused(lib, lib.heta_project(4, AT["a"], E4M3, 8, 8, AT["b"], F32, 8, 8, 0, None, AT["c"], F32, 8, 0.0, None), BAD, "")
    refused(lib, lib.heta_act_bwd(4, 8, hb.HETA_ACT_GELU, AT["a"], 8, AT["b"], 8, AT["c"], 8, None), BAD, "act")
