"""What heta_rms_norm, heta_linear, heta_muon_multi and their backward calls accept and refuse on the host, beyond what a single
spoiled argument shows: no device call is made here, the addresses belong to nothing."""
import ctypes
import os
import subprocess
import sys

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


@pytest.mark.parametrize("coarse", [0, 1])
def test_no_rows_of_8_bit_operands(lib, handle, coarse):
    """An empty tensor's address is null: 8-bit rows and their scales may be, where there are none."""
    a = dict(n_rows=0, d_in=64, d_out=48, inp=None, ld_in=64, in_scale=None, W=AT["b"], ld_w=64, w_scale=AT["h"], bias=AT["c"], out=None, ld_out=48,
             in_dt=E4M3, w_dt=E4M3, out_dt=BF16, act=hb.HETA_ACT_GELU, coarse_sums=coarse)
    assert lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**a)), None) == hb.HETA_OK
    refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**{**a, "w_scale": None})), None), BAD, "scales")
    refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**{**a, "n_rows": 1, "inp": AT["a"], "out": AT["d"]})), None), BAD, "scales")
    f = {**a, "in_dt": F32, "w_dt": F32, "out_dt": F32, "coarse_sums": 0, "w_scale": None}
    refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**{**f, "in_scale": AT["g"]})), None), BAD, "scales")


HYPER = (0.02, 0.9, 1, 0.0, 1e-7, 5)


def muon_item(rows, cols, **change):
    return hb._MuonItem(**{**dict(W=AT["a"], ld_w=cols, m=AT["b"], ld_m=cols, grad=AT["c"], ld_grad=cols, rows=rows, cols=cols, dt=F32, grad_dt=F32), **change})


@pytest.mark.parametrize("rows,cols", [(128, 17_000_000), (17_000_000, 128), (300, 17_000_000), (65, 2 ** 26 // 2 + 2 ** 20), (2, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2 ** 31 - 1, 1)])
def test_momentum_of_rows_whose_offsets_pass_32_bits(lib, handle, rows, cols):
    """Offsets from a tile's first row count in 32 bits: longer rows are refused."""
    refused(lib, lib.heta_muon_multi(handle, 1, ctypes.byref(muon_item(rows, cols)), *HYPER, None), UNSUPPORTED, "large")


OUT_OF_MEMORY = """
import ctypes, resource
from paper_2408_09697_amd import binding as hb
lib = hb.load_library()
n = 3_000_000
item = bytes(hb._MuonItem(W=0x10000000, ld_w=48, m=0x20000000, ld_m=48, grad=0x30000000, ld_grad=48, rows=64, cols=48, dt=hb.HETA_F32, grad_dt=hb.HETA_F32))
items = item * n
handle = ctypes.create_string_buffer(4096)
with open("/proc/self/statm") as f:
    size = int(f.read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (size + (64 << 20), resource.RLIM_INFINITY))
status = lib.heta_muon_multi(ctypes.addressof(handle), n, items, 0.02, 0.9, 1, 0.0, 1e-7, 5, None)
print(status, lib.heta_last_error().decode())
"""


def test_momentum_without_host_memory_for_its_lists():
    """An exception of the host's containers becomes a status (in a process of its own, whose address space ends 64 MB ahead)."""
    r = subprocess.run([sys.executable, "-c", OUT_OF_MEMORY], capture_output=True, text=True, timeout=100, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr[-500:]
    assert r.stdout.startswith(f"{hb.HETA_ERR_OOM} ") and "host allocation" in r.stdout, r.stdout


@pytest.mark.parametrize("change", [{"d_in": 70000, "d_out": 70000}, {"n_rows": 2 ** 31}])
def test_weight_gradients_too_large_are_refused_before_anything_else(lib, handle, change):
    a = dict(n_rows=100, d_in=64, d_out=48, dt=BF16, dw_dt=F32, act=hb.HETA_ACT_SILU, in_act=0)
    a.update(change)
    at = {name: 1 << 44 | i << 40 for i, name in enumerate(("inp", "W", "grad_out", "pre", "grad_pre", "grad_in", "dW", "dbias"))}  # 1 TB apart
    lds = dict(ld_inp=a["d_in"], ld_W=a["d_out"], ld_grad_out=a["d_out"], ld_pre=a["d_out"], ld_grad_pre=a["d_out"], ld_grad_in=a["d_in"], ld_dW=a["d_out"])
    refused(lib, lib.heta_linear_bwd(handle, ctypes.byref(hb._LinearBwdArgs(**a, **at, **lds)), None), UNSUPPORTED, "weight gradient")


NORM = dict(n=100, d=64, x=AT["a"], x_dt=F32, ld_x=64, res=AT["b"], ld_res=64, gamma=AT["c"], eps=1e-6, sum=AT["d"], ld_sum=64, out=AT["e"], out_dt=F32, ld_out=64,
            scale=None, rstd=AT["f"], stream=None)
NORM8 = dict(NORM, out_dt=E4M3, scale=AT["g"])


@pytest.mark.parametrize("base,change", [
    (NORM, {"gamma": AT["d"] + 64}), (NORM, {"gamma": AT["e"] + 99 * 256}), (NORM, {"rstd": AT["a"] + 256}), (NORM, {"rstd": AT["b"]}), (NORM, {"rstd": AT["c"] + 128}),
    (NORM, {"rstd": AT["d"] + 512}), (NORM, {"rstd": AT["e"] + 512}), (NORM8, {"scale": AT["a"]}), (NORM8, {"scale": AT["c"] + 252}), (NORM8, {"scale": AT["e"] + 64}),
    (NORM8, {"scale": AT["d"]}), (NORM8, {"scale": AT["f"] + 396})])
def test_norm_vectors_that_overlap(lib, base, change):
    refused(lib, lib.heta_rms_norm(*{**base, **change}.values()), BAD, "overlaps")


NORM_BWD = dict(g=1, n=100, d=64, x=AT["a"], x_dt=F32, ld_x=64, gamma=AT["c"], rstd=AT["d"], go=AT["e"], go_dt=F32, ld_go=64, gs=AT["f"], ld_gs=64, gx=AT["g"], ld_gx=64,
                gg=AT["h"], stream=None)


@pytest.mark.parametrize("change", [{"gg": AT["a"]}, {"gg": AT["c"] + 16}, {"gg": AT["d"] + 396}, {"gg": AT["e"] + 256}, {"gg": AT["f"]}, {"gg": AT["g"] + 99 * 256 + 252},
                                    {"gamma": AT["g"] + 64}, {"rstd": AT["g"] + 99 * 256}])
def test_norm_backward_vectors_that_overlap(lib, handle, change):
    refused(lib, lib.heta_rms_norm_bwd(*{**NORM_BWD, **change, "g": handle}.values()), BAD, "overlaps")


LINEAR = dict(n_rows=100, d_in=64, d_out=48, inp=AT["a"], ld_in=64, W=AT["b"], ld_w=48, bias=AT["c"], residual=AT["d"], ld_res=48, pre=AT["e"], ld_pre=48, out=AT["f"], ld_out=48,
              in_dt=F32, w_dt=F32, out_dt=F32, act=hb.HETA_ACT_GELU)
LINEAR8 = dict(LINEAR, in_dt=E4M3, w_dt=E4M3, ld_w=64, in_scale=AT["g"], w_scale=AT["h"])


@pytest.mark.parametrize("base,change", [
    (LINEAR, {"bias": AT["f"] + 192}), (LINEAR, {"bias": AT["e"] + 99 * 192}), (LINEAR8, {"in_scale": AT["f"]}), (LINEAR8, {"in_scale": AT["e"] + 1920}),
    (LINEAR8, {"w_scale": AT["f"] + 4}), (LINEAR8, {"w_scale": AT["e"]}), (LINEAR8, {"bias": AT["f"]})])
def test_linear_vectors_that_overlap(lib, handle, base, change):
    refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**{**base, **change})), None), BAD, "overlaps")


@pytest.mark.parametrize("flags", [4, 7, -1])
def test_momentum_flags(lib, handle, flags):
    refused(lib, lib.heta_muon_multi(handle, 1, ctypes.byref(muon_item(64, 48)), 0.02, 0.9, flags, 0.0, 1e-7, 5, None), BAD, "flags")


WIDE = 2 ** 31 - 1


def test_widths_near_2_to_the_31(lib, handle):
    """Column counters step by a workgroup's width and would pass 2^31."""
    far = {name: 1 << 44 | i << 40 for i, name in enumerate("abcdefgh")}  # 1 TB apart
    refused(lib, lib.heta_rms_norm(1, WIDE, far["a"], F32, WIDE, None, 0, None, 1e-6, None, 0, far["b"], F32, WIDE, None, None, None), UNSUPPORTED, "wide")
    refused(lib, lib.heta_rms_norm_bwd(handle, 1, WIDE, far["a"], F32, WIDE, None, far["b"], far["c"], F32, WIDE, None, 0, far["d"], WIDE, far["e"], None), UNSUPPORTED, "wide")
    for d_in, d_out in ((1, WIDE), (WIDE, 1)):
        a = dict(n_rows=1, d_in=d_in, d_out=d_out, inp=far["a"], ld_in=d_in, W=far["b"], ld_w=d_out, out=far["c"], ld_out=d_out, in_dt=BF16, w_dt=BF16, out_dt=BF16)
        refused(lib, lib.heta_linear(handle, ctypes.byref(hb._LinearArgs(**a)), None), UNSUPPORTED, "wide")
        a = dict(n_rows=1, d_in=d_in, d_out=d_out, dt=BF16, dw_dt=BF16, inp=far["a"], ld_inp=d_in, W=far["b"], ld_W=d_out, grad_out=far["c"], ld_grad_out=d_out, grad_in=far["d"],
                 ld_grad_in=d_in, dW=far["e"], ld_dW=d_out, dbias=far["f"])
        refused(lib, lib.heta_linear_bwd(handle, ctypes.byref(hb._LinearBwdArgs(**a)), None), UNSUPPORTED, "wide")
        refused(lib, lib.heta_linear_pack_e4m3(far["a"], F32, d_out, d_in, d_out, far["b"], d_in, far["c"], None), UNSUPPORTED, "wide")
