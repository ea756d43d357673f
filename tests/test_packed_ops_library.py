"""What the built libraries' kernels of the operations on packed sequences keep to: no scratch memory, room for a second workgroup, and
the distances of the MFMAs that are inline assembly, which the compiler does not know."""
import re
import subprocess

import pytest

from test_library_abi import _code_objects, _kernel_scratch, _llvm_tool, _near_mfmas

LIBRARIES = pytest.mark.parametrize("elem", ["bf16", "fp16"])


@LIBRARIES
def test_kernels_use_no_scratch_memory(elem, tmp_path):
    from paper_2110_13005_amd import build as BLD
    names = ("attn_packed_", "token_logprobs", "policy_loss", "preference_loss", "distill_loss", "weighted_sum")
    scratch = {k: v for k, v in _kernel_scratch(BLD.VARIANTS[elem][0], tmp_path).items() if any(n in k for n in names)}
    assert all(any(n in k for k in scratch) for n in names)
    assert not {k: v for k, v in scratch.items() if v}


@LIBRARIES
def test_two_workgroups_share_a_cu_where_they_should(elem, tmp_path):
    """The forward and dQ kernels up to 128 columns: half of a SIMD's 512 registers per lane and of 160 KB of LDS at most."""
    from paper_2110_13005_amd import build as BLD
    readelf, seen = _llvm_tool("llvm-readelf"), 0
    for obj in _code_objects(BLD.VARIANTS[elem][0], tmp_path):
        notes = subprocess.run([readelf, "--notes", str(obj)], capture_output=True, text=True, check=True).stdout
        for kernel in re.split(r"^ +- \.agpr_count:", notes, flags=re.M)[1:]:
            name = re.search(r"\.name: +\S*?attn_packed_(fwd|bwd_dq)_kernelILi(\d+)E", kernel)
            if name and int(name.group(2)) <= 128:
                seen += 1
                assert int(re.search(r"\.vgpr_count: +(\d+)", kernel).group(1)) <= 256, name.group(0)
                assert int(re.search(r"\.group_segment_fixed_size: +(\d+)", kernel).group(1)) <= 80 * 1024, name.group(0)
    assert seen >= 4


@LIBRARIES
def test_mfma_distances_along_every_path(elem, tmp_path):
    """In the kernels that form dK and dV: two wait states, and twelve or two MFMAs, whichever way the kernel takes."""
    from paper_2110_13005_amd import build as BLD
    objdump, kernels = _llvm_tool("llvm-objdump"), 0
    for obj in _code_objects(BLD.VARIANTS[elem][0], tmp_path):
        text = subprocess.run([objdump, "-d", "--no-show-raw-insn", str(obj)], capture_output=True, text=True, check=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\S*attn_packed_bwd_(?:dkdv|both)\S*)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, flags=re.M | re.S):
            kernels += 1
            near = _near_mfmas(body)
            assert not near, (name, [(hex(at), op, operands) for at, op, operands, _ in near[:4]])
    assert kernels >= 5
