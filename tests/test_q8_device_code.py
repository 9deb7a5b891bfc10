"""What the compiler made of the kernels for 8-bit products, for activations that keep 8 bits and for sampling, read from the gfx950 assembly of the shipped sources
built with the shipped flags: nothing spills, the tiles' loads pass registers by and are waited for by count, the accumulators stay where the matrix
cores write them, and kernels that count on two blocks to a CU have the registers for that."""
import os
import re
import subprocess

import pytest

from paper_1909_07729_amd import build

SOURCES = ["ktanh_q8_product.hip", "ktanh_q8_few.hip", "ktanh_q8_rows.hip", "ktanh_keep8.hip", "ktanh_sample.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: (code, registers, spilled, LDS)} of every kernel."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    tmp, procs, out = tmp_path_factory.mktemp("asm"), [], {}
    for src in SOURCES:
        dst = str(tmp / (src + ".s"))
        cmd = [hipcc, *flags, "-S", "--cuda-device-only", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, os.path.join(build.CSRC, src), "-o", dst]
        procs.append((dst, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE)))
    for dst, p in procs:
        _, err = p.communicate(timeout=600)
        assert p.returncode == 0, err.decode()
        text = open(dst).read()
        parts = re.split(r"^(_Z\w+):", text, flags=re.M)
        code = {n: body[:body.index(".Lfunc_end")] for n, body in zip(parts[1::2], parts[2::2]) if "s_endpgm" in body}
        for entry in re.split(r"^  - \.agpr_count:", text, flags=re.M)[1:]:
            name = re.search(r"\.name:\s+(\S+)", entry).group(1)
            fields = ("vgpr_count", "vgpr_spill_count", "group_segment_fixed_size", "private_segment_fixed_size")
            out[name] = code[name], *(int(re.search(rf"\.{field}:\s+(\d+)", entry).group(1)) for field in fields)
    return out


def _of(kernels, name):
    found = {n: k for n, k in kernels.items() if name in n}
    assert found, name
    return found


def test_no_kernel_spills(kernels):
    assert all(spilled == 0 and private == 0 for _, _, spilled, _, private in kernels.values())


def _loop(code):
    """The code of the loop over tiles: from the label that is jumped back to, to the jump."""
    for label, body in re.findall(r"^(\.LBB\d+_\d+):[^\n]*\n(.*?)(?=^\.LBB\d+_\d+:|\Z)", code, flags=re.M | re.S):
        back = re.search(rf"s_cbranch_\w+ {re.escape(label)}\b", body)
        if back and "v_mfma_i32_32x32x32_i8" in body[:back.start()]:
            return body[:back.start()]
    raise AssertionError("no loop")


def test_the_loop_over_tiles(kernels):
    """One counted wait and one barrier to a tile; loads that pass registers by, of all tiles of the ring but one in flight; no accumulator moves."""
    for n, (code, *_) in _of(kernels, "q8_tile_kernel").items():
        over, across, places = (int(i) for i in re.search(r"q8_tile_kernelILj(\d+)ELj(\d+)ELj(\d+)", n).groups())
        loop = _loop(code)
        loads = (over + across) // 32
        assert loop.count("global_load_lds_dwordx4") == loads, n
        assert re.findall(r"vmcnt\((\d+)\)", loop) == [str(loads * (places - 2))], n
        assert loop.count("s_barrier") == 1 and loop.count("v_mfma_i32_32x32x32_i8") == 4 * over * across // 4096, n
        assert "accvgpr" not in loop and not re.search(r"\bglobal_load_dword|\bglobal_store|buffer_|scratch_", loop), n


def test_room_for_two_blocks(kernels):
    """512 registers a lane and SIMD, 160 KB of LDS a CU."""
    for n, (_, registers, _, lds, _) in _of(kernels, "q8_tile_kernel").items():
        over, across, places = (int(i) for i in re.search(r"q8_tile_kernelILj(\d+)ELj(\d+)ELj(\d+)", n).groups())
        if places * (over + across) * 128 <= 81920:
            assert registers <= 256 and lds <= 81920, n
    for name in ("sample_bins_kernel", "sample_answer_kernel"):
        for n, (_, registers, _, lds, _) in _of(kernels, name).items():
            assert registers <= 64 and lds <= 81920, n


def test_rows_behind_an_activation_take_few_registers(kernels):
    """Eight vectors of a lane are held, one of them worked on."""
    for n, (_, registers, _, _, _) in _of(kernels, "q8_rows_kernel").items():
        assert registers <= 128, (n, registers)
