"""Registers, LDS and scratch of the built kernels over a 4-bit cache, of the keys' weights and of eviction, against what their
launch rules and comments count on (read from the kernel descriptors of the library, host only)."""
import re

import pytest

from paper_2602_04361_amd import sparvar as sv
from test_kernel_registers import code_objects
from test_q8_kernel_resources import LDS_CU, descriptors

NAMES = r"attn_q4_(few_|rows_)?kernelI|kv_(de)?quantize_q4_kernelI|key_weights_(few_)?kernelI|kv_evict_kernelI"


@pytest.fixture(scope="module")
def kernels():
    with open(sv.LIB_PATH, "rb") as f:
        data = f.read()
    found = {}
    for elf in code_objects(data):
        found.update(descriptors(elf))
    return {n: v for n, v in found.items() if re.search(NAMES, n)}


# waves of a workgroup, workgroups a CU (of four SIMDs of 512 registers a lane)
@pytest.mark.parametrize("kernel,waves,workgroups", [
    (r"attn_q4_kernelILi128ELi1ELi1E\w*13SparseRowsSrc", 1, 5), (r"attn_q4_kernelILi64ELi1ELi1E\w*13SparseRowsSrc", 1, 10),
    (r"attn_q4_kernelILi128ELi2ELi1E\w*13SparseRowsSrc", 2, 4), (r"attn_q4_kernelILi64ELi2ELi1E\w*13SparseRowsSrc", 2, 6),
    (r"attn_q4_kernelILi64ELi2ELi2E\w*13SparseRowsSrc", 4, 3), (r"attn_q4_kernelILi128ELi2ELi2E\w*13SparseRowsSrc", 4, 2),
    (r"attn_q4_kernelILi64ELi2ELi4E\w*13SparseRowsSrc", 8, 1), (r"attn_q4_kernelILi128ELi2ELi4E\w*13SparseRowsSrc", 8, 1),
    (r"attn_q4_kernelILi128ELi8ELi1E\w*12DenseRowsSrc", 8, 1), (r"attn_q4_kernelILi128ELi4ELi1E\w*12DenseRowsSrc", 4, 2),
    (r"attn_q4_kernelILi128ELi4ELi2E\w*12DenseRowsSrc", 8, 1), (r"attn_q4_kernelILi128ELi2ELi4E\w*12DenseRowsSrc", 8, 1),
    (r"attn_q4_kernelILi64ELi8ELi1E\w*12DenseRowsSrc", 8, 1), (r"attn_q4_kernelILi64ELi4ELi1E\w*12DenseRowsSrc", 4, 3),
    (r"attn_q4_rows_kernelILi128E", 4, 2), (r"attn_q4_rows_kernelILi64E", 4, 3),
    (r"attn_q4_few_kernelILi128E", 4, 3), (r"attn_q4_few_kernelILi64E", 4, 5),
    # (bf16 and 4-bit keys: of 256 keys two workgroups, of 128 three)
    (r"18key_weights_kernelILNS0_4KeysE0ELi128ELi4ELi1ELi2E", 4, 2), (r"18key_weights_kernelILNS0_4KeysE2ELi128ELi4ELi1ELi2E", 4, 2),
    (r"18key_weights_kernelILNS0_4KeysE0ELi128ELi4ELi1ELi1E", 4, 3), (r"18key_weights_kernelILNS0_4KeysE2ELi128ELi4ELi1ELi1E", 4, 3),
    (r"18key_weights_kernelILNS0_4KeysE1ELi128ELi4ELi1ELi1E", 4, 2), (r"18key_weights_kernelILNS0_4KeysE1ELi128ELi1ELi4ELi1E", 4, 1),
    (r"kv_evict_kernelILi12E", 16, 1), (r"kv_evict_kernelILi2E", 16, 2)])
def test_workgroups_per_cu(kernels, kernel, waves, workgroups):
    got = [v for n, v in kernels.items() if re.search(kernel, n)]
    assert len(got) == 1, kernel
    vgprs, lds, _ = got[0]
    assert (512 // vgprs) * 4 >= waves * workgroups, vgprs
    assert lds * workgroups <= LDS_CU, lds


def test_scratch(kernels):
    """None, in any of them."""
    assert len(kernels) == 20 + 4 + 4 + 22 + 6 + 4
    assert {n: s for n, (_, _, s) in kernels.items() if s} == {}
