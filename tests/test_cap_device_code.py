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


def _writes_before_loads_arrive(code):
    """Blocks of the code with four or more wide LDS writes (tensors that leave through LDS) that some path enters with a direct load on its way."""
    blocks, starts = [], {}
    for line in code.splitlines():
        text = line.split(";")[0].strip()
        label = re.match(r"(\.LBB\d+_\d+):", text)
        if label or not blocks:
            blocks.append([])
        if label:
            starts[label.group(1)] = len(blocks) - 1
        elif text:
            blocks[-1].append(text)
            if re.match(r"s_c?branch", text):
                blocks.append([])
    follows = []
    for i, block in enumerate(blocks):
        last = block[-1] if block else ""
        to = [i + 1] if i + 1 < len(blocks) and not re.match(r"s_(branch|endpgm)", last) else []
        jump = re.match(r"s_c?branch\w*\s+(\S+)", last)
        follows.append(to + ([starts[jump.group(1)]] if jump else []))

    def run(block, coming):
        """(whether a load may be on its way behind the block, whether it is at a tensor's write)"""
        writes = [i for i, text in enumerate(block) if re.match(r"ds_write\w*_b(64|128)", text)]
        early = False
        for i, text in enumerate(block):
            if text.startswith("global_load_lds"):
                coming = True
            elif re.match(r"s_waitcnt.*vmcnt\(0\)", text):
                coming = False
            elif i in writes and len(writes) >= 4 and coming:
                early = True
        return coming, early
    entered, work, found = {0: False}, [0], set()
    while work:
        i = work.pop()
        coming, early = run(blocks[i], entered[i])
        if early:
            found.add(i)
        for to in follows[i]:
            if to not in entered or coming and not entered[to]:
                entered[to] = coming
                work.append(to)
    return found


def test_values_have_arrived_before_their_place_is_written(kernels):
    """Blocks of 128 keys keep their values in LDS, and write their gradients through that place.  Where no query sees the block there is no tile
    whose wait would cover the values' loads; a load that lands behind the writes would be stored as a gradient."""
    found = _of(kernels, "cap_dkdv_kernel")
    plain = {n: code for n, (code, _, _) in found.items() if "Lb0EE" in n}
    assert len(plain) == 2
    for n, code in plain.items():
        assert not _writes_before_loads_arrive(code), n


def test_the_reading_of_late_loads_finds_them():
    """The check above on code that has the fault on one of two paths, and on code that waits on both."""
    writes = "\n".join(["  ds_write_b64 v1, v[2:3]"] * 4)
    code = "  global_load_lds_dwordx4 v[0:1], off\n  s_cbranch_scc1 .LBB0_2\n  s_waitcnt vmcnt(0)\n.LBB0_2:\n{}" + writes + "\n  s_endpgm\n"
    assert _writes_before_loads_arrive(code.format("")) and not _writes_before_loads_arrive(code.format("  s_waitcnt vmcnt(0) lgkmcnt(0)\n"))
