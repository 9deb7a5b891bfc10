"""What the compiler made of the capped attention's kernels, read from the gfx950 assembly of the shipped sources built with the shipped
flags: tiles come by direct loads that nothing but the step's own wait waits for, operands by transposing reads, and
registers leave room for the wavefronts that the design counts on."""
import os
import re
import subprocess

import pytest

from paper_1909_07729_amd import build

SOURCES = ["ktanh_cap_forward.hip", "ktanh_cap_backward.hip", "ktanh_cap_decode.hip", "ktanh_cap_append.hip"]


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: (code, registers, spilled)} of every kernel."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    tmp, procs, out = tmp_path_factory.mktemp("asm"), [], {}
    for src in SOURCES:
        dst = str(tmp / (src + ".s"))
        cmd = [hipcc, *flags, "-S", "--cuda-device-only", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
               os.path.join(build.CSRC, src), "-o", dst]
        procs.append((dst, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.PIPE)))
    for dst, p in procs:
        _, err = p.communicate(timeout=600)
        assert p.returncode == 0, err.decode()
        text = open(dst).read()
        parts = re.split(r"^(_Z\w+):", text, flags=re.M)
        code = {n: body[:body.index(".Lfunc_end")] for n, body in zip(parts[1::2], parts[2::2]) if "s_endpgm" in body}
        for entry in re.split(r"^  - \.agpr_count:", text, flags=re.M)[1:]:
            name = re.search(r"\.name:\s+(\S+)", entry).group(1)
            out[name] = code[name], *(int(re.search(rf"\.{field}:\s+(\d+)", entry).group(1)) for field in ("vgpr_count", "vgpr_spill_count"))
    return out


def _of(kernels, name):
    found = {n: k for n, k in kernels.items() if name in n}
    assert found, name
    return found


def _blocks(code):
    return re.split(r"^\.LBB\d+_\d+:", code, flags=re.M)


def test_no_kernel_spills(kernels):
    assert all(spilled == 0 for _, _, spilled in kernels.values())


def test_tiles_come_by_direct_loads_and_transposing_reads(kernels):
    for name in ("cap_forward_kernel", "cap_dq_kernel", "cap_dkdv_kernel"):
        for n, (code, _, _) in _of(kernels, name).items():
            assert "global_load_lds_dwordx4" in code and "ds_read_b64_tr_b16" in code and "v_mfma_f32_32x32x16_bf16" in code, n


def test_nothing_waits_for_the_next_tile(kernels):
    """In the code of a tile (the products and all between them) no instruction waits for memory: the next tile's loads are in flight."""
    for name in ("cap_forward_kernel", "cap_dq_kernel", "cap_dkdv_kernel"):
        for n, (code, _, _) in _of(kernels, name).items():
            tiles = [b for b in _blocks(code) if b.count("v_mfma_f32_32x32x16_bf16") >= 4]
            assert tiles, n
            assert not any("vmcnt" in b for b in tiles), n


def test_registers_leave_room_for_the_wavefronts(kernels):
    """512 registers a lane and SIMD: three wavefronts of the forward's blocks of 128 rows, two of everything else that holds tiles."""
    for n, (_, registers, _) in _of(kernels, "cap_forward_kernel").items():
        assert registers <= (256 if re.search(r"Lb1EEEv", n) else 168), (n, registers)
    for name in ("cap_dq_kernel", "cap_dkdv_kernel", "cap_decode_kernel"):
        for n, (_, registers, _) in _of(kernels, name).items():
            assert registers <= 256, (n, registers)


def test_what_is_read_once_is_read_with_the_streaming_hint(kernels):
    for name in ("cap_decode_kernel", "cap_append_kernel"):
        for n, (code, _, _) in _of(kernels, name).items():
            assert re.search(r"global_load_dwordx4 .* nt", code), n
