"""Kernels of the product template keep within their registers, by the metadata that the compiler left in the library built here.

Where one of them spilled, copies of live values were placed in front of the instruction that brings masked lanes back, and those lanes read the
next tile from stale addresses (see heta_tiles.h)."""
import os
import re
import struct
import subprocess

import pytest

from paper_2408_09697_amd import binding as hb

READELF = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-readelf")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def device_images(path):
    """The gfx950 code objects of a library: entries of its offload bundles (offset, size, length of the name, name)."""
    with open(path, "rb") as f:
        data = f.read()
    at = data.find(MAGIC)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + length] and size > 0:
                yield data[at + offset:at + offset + size]
            p += 24 + length
        at = data.find(MAGIC, at + 24)


@pytest.mark.skipif(not os.path.exists(READELF), reason="llvm-readelf is not installed")
def test_products_do_not_spill(tmp_path):
    seen, spilled = 0, []
    for i, image in enumerate(device_images(hb.LIB_PATH)):
        f = tmp_path / f"{i}.co"
        f.write_bytes(image)
        notes = subprocess.run([READELF, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
        for kernel in re.split(r"\n\s+- \.agpr_count:", notes)[1:]:
            name = re.search(r"\.name:\s+(\S+)", kernel).group(1)
            if "tile_gemm_kernel" not in name:
                continue
            seen += 1
            if int(re.search(r"\.vgpr_spill_count:\s+(\d+)", kernel).group(1)) or int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", kernel).group(1)):
                spilled.append(name)
    assert seen >= 40 and not spilled, spilled


OBJDUMP = os.path.join(os.path.dirname(READELF), "llvm-objdump")


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="llvm-objdump is not installed")
def test_m0_is_written_a_wait_state_before_loads_into_lds(tmp_path):
    """gfx9 wants one between a scalar write of M0 and a load that takes its LDS address from there."""
    loads = 0
    for i, image in enumerate(device_images(hb.LIB_PATH)):
        if b"gemm" not in image:
            continue
        f = tmp_path / f"{i}.co"
        f.write_bytes(image)
        before = ""
        with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(f)], stdout=subprocess.PIPE, text=True) as p:
            for line in p.stdout:
                op = line.split("//")[0].strip()
                if op.startswith("global_load_lds"):
                    loads += 1
                    assert not re.match(r"s_\S+ m0,", before), f"{before}; {op}"
                if op:
                    before = op
    assert loads > 1000
