"""Registers, LDS and scratch of the built kernels over an 8-bit cache, against what their launch rules and comments count on
(read from the kernel descriptors of the library, host only)."""
import re
import struct

import pytest

from paper_2602_04361_amd import sparvar as sv
from test_kernel_registers import code_objects

LDS_CU = 160 * 1024


def descriptors(elf):
    """Mangled kernel name -> (VGPRs of a wave, LDS bytes of a workgroup, scratch bytes of a lane)."""
    shoff, = struct.unpack_from("<Q", elf, 40)
    entsize, num = struct.unpack_from("<HH", elf, 58)
    heads = [struct.unpack_from("<IIQQQQIIQQ", elf, shoff + i * entsize) for i in range(num)]
    out = {}
    for _, kind, _, _, offset, size, link, _, _, ent in heads:
        if kind != 11:  # dynamic symbols
            continue
        for i in range(0, size, ent):
            name, _, _, _, value, _ = struct.unpack_from("<IBBHQQ", elf, offset + i)
            start = heads[link][4] + name
            text = elf[start:elf.index(b"\0", start)].decode()
            if not text.endswith(".kd"):
                continue
            _, _, _, addr, base, _, _, _, _, _ = next(h for h in heads if h[1] == 1 and h[3] <= value < h[3] + h[5])
            at = base + value - addr
            lds, scratch = struct.unpack_from("<II", elf, at)
            out[text[:-3]] = (((struct.unpack_from("<I", elf, at + 48)[0] & 63) + 1) * 8, lds, scratch)
    return out


@pytest.fixture(scope="module")
def kernels():
    with open(sv.LIB_PATH, "rb") as f:
        data = f.read()
    found = {}
    for elf in code_objects(data):
        found.update(descriptors(elf))
    return {n: v for n, v in found.items() if "_q8_" in n}


def the(kernels, pattern):
    got = {n: v for n, v in kernels.items() if re.search(pattern, n)}
    assert len(got) == 1, sorted(got)
    return next(iter(got.values()))


# waves of a workgroup, workgroups a CU (of four SIMDs of 512 registers a lane)
@pytest.mark.parametrize("kernel,waves,workgroups", [
    (r"attn_q8_kernelILi128ELi2ELi1E\w*11SparseQ8Src", 2, 4), (r"attn_q8_kernelILi64ELi2ELi1E\w*11SparseQ8Src", 2, 6),
    (r"attn_q8_kernelILi64ELi2ELi2E\w*11SparseQ8Src", 4, 3), (r"attn_q8_kernelILi128ELi2ELi2E\w*11SparseQ8Src", 4, 2),
    (r"attn_q8_kernelILi64ELi2ELi4E\w*11SparseQ8Src", 8, 1), (r"attn_q8_kernelILi128ELi2ELi4E\w*11SparseQ8Src", 8, 1),
    (r"attn_q8_kernelILi128ELi8ELi1E\w*10DenseQ8Src", 8, 1), (r"attn_q8_kernelILi128ELi4ELi1E\w*10DenseQ8Src", 4, 2),
    (r"attn_q8_kernelILi128ELi4ELi2E\w*10DenseQ8Src", 8, 1), (r"attn_q8_kernelILi128ELi2ELi4E\w*10DenseQ8Src", 8, 1),
    (r"attn_q8_kernelILi64ELi8ELi1E\w*10DenseQ8Src", 8, 1), (r"attn_q8_kernelILi64ELi4ELi1E\w*10DenseQ8Src", 4, 3),
    (r"attn_q8_rows_kernelILi128E", 4, 2), (r"attn_q8_rows_kernelILi64E", 4, 3)])
def test_workgroups_per_cu(kernels, kernel, waves, workgroups):
    vgprs, lds, _ = the(kernels, kernel)
    assert (512 // vgprs) * 4 >= waves * workgroups, vgprs
    assert lds * workgroups <= LDS_CU, lds


def test_scratch(kernels):
    """None, but for up to four words a lane where two or four sets of waves fill the registers at d = 128."""
    assert len(kernels) == 22
    for name, (_, _, scratch) in kernels.items():
        sets = re.search(r"attn_q8_kernelILi128ELi2ELi[24]E", name)
        assert scratch <= (16 if sets else 0), name
