"""What the built libraries' kernels of the step's single operations keep to: no scratch memory, and the distances of the MFMAs that
are inline assembly, which the compiler does not know."""
import re
import subprocess

import pytest

from test_library_abi import _code_objects, _kernel_scratch, _llvm_tool, _registers


@pytest.mark.parametrize("elem", ["bf16", "fp16"])
def test_kernels_use_no_scratch_memory(elem, tmp_path):
    from paper_2110_13005_amd import build as BLD
    names = ("embedding_", "qk_", "dropout_", "fp8_")
    scratch = {k: v for k, v in _kernel_scratch(BLD.VARIANTS[elem][0], tmp_path).items() if any(n in k for n in names)}
    assert len(scratch) > 60
    assert not {k: v for k, v in scratch.items() if v}


@pytest.mark.parametrize("elem", ["bf16", "fp16"])
def test_scaled_mfmas_keep_their_distances(elem, tmp_path):
    """In the 256 x 256 kernel of the 8-bit product: two instructions between a vector instruction and an MFMA that reads its
    result, in program order, and 48 idle cycles between the last MFMA in front of the epilogue and the first instruction
    that reads an accumulator."""
    from paper_2110_13005_amd import build as BLD
    objdump, kernels = _llvm_tool("llvm-objdump"), 0
    for obj in _code_objects(BLD.VARIANTS[elem][0], tmp_path):
        text = subprocess.run([objdump, "-d", "--no-show-raw-insn", str(obj)], capture_output=True, text=True, check=True).stdout
        for name, body in re.findall(r"<(\S*gemm_fp8_big_kernel\S*)>:\n(.*?)\n\n", text + "\n\n", flags=re.S):
            kernels += 1
            code = [line.split("//")[0].strip() for line in body.split("\n") if line.strip()]
            mfmas = [i for i, line in enumerate(code) if line.startswith("v_mfma")]
            assert len(mfmas) == 256, name
            for i in mfmas:
                operands = code[i].split(None, 1)[1].split(", ")
                reads = set().union(*(_registers(o) for o in operands[1:6]))
                for back in (1, 2):
                    line = code[i - back]
                    if line.startswith("v_") and not line.startswith("v_mfma"):
                        assert not reads & _registers(line.split(None, 1)[1].split(", ")[0]), (name, code[i - back], code[i])
            # behind the last MFMA: nothing touches an accumulator until the idle cycles are over
            idle = 0
            for line in code[mfmas[-1] + 1:]:
                if line.startswith("s_nop"):
                    idle += int(line.split()[1]) + 1
                touched = set().union(*(_registers(o) for o in line.split(None, 1)[1].split(", "))) if " " in line else set()
                if any(kind == "a" for kind, _ in touched):
                    break
            assert idle >= 48, (name, idle)
    assert kernels == 5
