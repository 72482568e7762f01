"""What the kernels' sources have to say to the compiler, and what it has to say of them (CPU only)."""
import glob
import os
import re

import pytest

from paper_2605_16867_amd import build


def _asm_statements():
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.hip")) + glob.glob(os.path.join(build.CSRC, "*.h"))):
        for m in re.finditer(r"\basm\b[^;\"]*\((.*?)\);", open(path).read(), flags=re.S):
            yield os.path.basename(path), m.group(1)


def test_assembly_names_its_special_registers():
    """A register that a statement writes by name is one that the compiler must not keep anything in; a load into shared memory has its place in m0
    from the compiler or sets it, and says so."""
    seen = 0
    for path, text in _asm_statements():
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text.split("::")[0].split(" : ")[0]))
        for name in ("m0", "vcc", "exec", "scc"):
            if re.search(rf"\b[sv]_\w+ {name}\b", code):
                assert f'"{name}"' in text.rsplit(":", 1)[1], (path, text)
        if "_lds_" in code:
            seen += 1
            assert '"{m0}"' in text or '"m0"' in text, (path, text)
    assert seen >= 2


def test_assembly_waits_for_scalars_of_the_vector_unit():
    """A scalar register that the vector unit has written may be read by memory's five wait states later; nothing but the statement itself sees to
    that where it has both."""
    seen = 0
    for path, text in _asm_statements():
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', text.split("::")[0]))
        constraints = re.findall(r'"([^"]*)"\s*\(', text)
        states = 0
        for line in code.replace("\\t", "").split("\\n"):
            if re.match(r"(global|buffer|flat|scratch)_", line):
                operands = [int(i) for i in re.findall(r"%(\d)", line)]
                if any(constraints[i] == "s" for i in operands):
                    seen += 1
                    assert states >= 5, (path, text)
            nop = re.match(r"s_nop (\d+)", line)
            states += int(nop.group(1)) + 1 if nop else 1
    assert seen >= 1


def _remarks(*kernels):
    text = "linear.hip:20:1: warning: of something else\n"
    for name, spilled, scratch in kernels:
        for line in (f"Function Name: {name}", "    VGPRs: 202", f"    ScratchSize [bytes/lane]: {scratch}", "    SGPRs Spill: 96",
                     f"    VGPRs Spill: {spilled}", "    LDS Size [bytes/block]: 163840"):
            text += f"linear.hip:479:1: remark: {line} [-Rpass-analysis=kernel-resource-usage]\n  479 | {{\n      | ^\n"
    return text


def test_a_build_with_spilled_sums_fails():
    tiles, other = "_ZN2gr14k_linear_tilesIDF16bLi256EEEvNS0_10LinearArgsE", "_ZN2gr7k_routeIfEEvNS_9RouteArgsE"
    build.check_spills(_remarks((other, 4, 16), (tiles, 0, 0), (tiles, 0, 0)))
    for bad in (((tiles, 0, 0), (tiles, 1, 0)), ((tiles, 0, 8), (other, 0, 0)), ((other, 0, 0),), ()):
        with pytest.raises(RuntimeError, match="k_linear_tiles"):
            build.check_spills(_remarks(*bad))
    with pytest.raises(RuntimeError, match="no word of"):
        build.check_spills(_remarks((tiles, 0, 0)).replace("VGPRs Spill", "spilled"))
