"""What the compiler makes of branches that mask lanes, in the kernels that hold most registers (assembly of this library's own
sources, no GPU).

A branch whose condition differs between lanes clears their bits of `exec` and, where none is left, jumps over its body to the join, which
restores `exec`.  A vector instruction in front of that restoring is carried out for the lanes that took the body only; by a wavefront that jumped,
for none.  In merit_delta_chunks (fp32, rows off 16 bytes, states kept) the compiler once put the copy of a register that all
lanes use later there, and wavefronts that had jumped went on with an old value."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_1911_03458_amd import build

SOURCES = [s for s in build.SOURCES if re.match(r"(delta|block_norm)_\w+\.hip", s)]
MASK_BACK = re.compile(r"s_or_b64 exec, exec|s_or_saveexec_b64|s_andn2_saveexec_b64")
VECTOR = re.compile(r"v_(?!readlane|writelane|readfirst|cmp)|scratch_|buffer_|ds_|global_")


def early_copies(assembly):
    """(function, line, instructions) of joins reached by a jump with vector instructions in front of the mask's restoring"""
    lines = assembly.split("\n")
    targets = set(re.findall(r"s_cbranch_execz (\.LBB\S+)", assembly))
    found, function, before = [], None, None
    for number, line in enumerate(lines, 1):
        label = re.match(r"(_Z\S+|\.LBB\S+):", line)
        if label:
            if label.group(1).startswith("_Z"):
                function = label.group(1)
            before = [] if label.group(1) in targets else None
        elif line.startswith("; %bb"):
            before = None
        elif before is not None and line.startswith("\t") and not line.strip().startswith((".", ";")):
            ins = line.strip()
            if MASK_BACK.match(ins):
                vector = [i for i in before if VECTOR.match(i)]
                if vector:
                    found.append((function, number, vector))
                before = None
            elif re.match(r"s_cbranch|s_branch|s_endpgm", ins):
                before = None
            else:
                before.append(ins)
    return found


def test_the_search_sees_one():
    text = "_Z1fv:\n\ts_and_saveexec_b64 s[0:1], vcc\n\ts_cbranch_execz .LBB0_2\n; %bb.1:\n\tv_add_u32_e32 v1, 1, v1\n.LBB0_2:\n"
    assert early_copies(text + "\tv_mov_b32_e32 v15, v185\n\ts_or_b64 exec, exec, s[0:1]\n") == [("_Z1fv", 8, ["v_mov_b32_e32 v15, v185"])]
    assert not early_copies(text + "\ts_or_b64 exec, exec, s[0:1]\n\tv_mov_b32_e32 v15, v185\n")


def test_no_copy_in_front_of_a_mask(tmp_path):
    try:
        command = build.compile_command()
    except RuntimeError:
        pytest.skip("no hipcc")
    assert len(SOURCES) == 6

    def assembly(source):
        out = tmp_path / (source + ".s")
        r = subprocess.run(command + ["--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return out.read_text()

    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        for source, text in zip(SOURCES, pool.map(assembly, SOURCES)):
            assert text.count("s_cbranch_execz") > 10, source
            assert not early_copies(text), source
