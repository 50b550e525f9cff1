"""What the training-step kernels' code must and must not hold, read from the assembly that the library's compiler and flags make of
their sources; no GPU.  The library allocates nothing, so none of them keeps anything in scratch memory, which the runtime would have to
allocate.  And the parts that a scalar load adds up to its address are whole words: it leaves out the lowest two bits of each."""
import os
import re
import subprocess

import pytest

from paper_2409_02423_amd import build

SOURCES = [s for s in build.SOURCES if os.path.basename(s).startswith("zt_")]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    work = tmp_path_factory.mktemp("asm")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    running = []
    for source in SOURCES:
        out = str(work / (os.path.basename(source) + ".s"))
        running.append((os.path.basename(source), out, subprocess.Popen(
            [build.HIPCC] + flags + ["-S", "--cuda-device-only", source, "-o", out], stderr=subprocess.DEVNULL)))
    texts = {}
    for name, out, process in running:
        assert process.wait() == 0, name
        with open(out) as f:
            texts[name] = f.read()
    return texts


@pytest.mark.parametrize("source, least", (("zt_step.hip", 12), ("zt_norm.hip", 12 * 8), ("zt_norm_backward.hip", 24 * 4)))
def test_no_kernel_uses_scratch(assembly, source, least):
    kernels = re.findall(r"\.amdhsa_kernel (\S+)\n(.*?)\.end_amdhsa_kernel", assembly[source], flags=re.S)
    assert len(kernels) >= least
    for name, meta in kernels:
        assert re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", meta).group(1) == "0", name


def test_scalar_loads_add_up_whole_words(assembly):
    written, loads = {}, 0
    for line in assembly["zt_step.hip"].splitlines():
        line = line.strip()
        m = re.match(r"s_load_dword\w*\s+\S+ s\[\d+:\d+\], (s\d+)(?: offset:(\w+))?$", line)
        if m:
            loads += 1
            how = written.get(m.group(1), "")
            shift = re.match(r"s_lshl_b32 s\d+, s\d+, (\d+)$", how)
            assert shift and int(shift.group(1)) >= 2, (line, how)
            assert int(m.group(2) or "0", 0) % 4 == 0, line
        m = re.match(r"s_\w+\s+(s\d+)\b", line)
        if m:
            written[m.group(1)] = line
    assert loads > 0


def test_rows_in_lds_take_what_a_workgroup_has_of_them(assembly):
    """Where a row's values lie in LDS the backward kernel asks for its workgroup's lanes, 16-byte vectors as fp32 for each, and little beside."""
    kernels = re.findall(r"\.amdhsa_kernel (\S*norm_backward_kernel\S+)\n(.*?)\.end_amdhsa_kernel", assembly["zt_norm_backward.hip"], flags=re.S)
    seen = 0
    for name, meta in kernels:
        # type, LayerNorm, post, channel gate, vectors a lane (n..: short rows; 0: any width), lanes, what registers hold (2: all)
        dtype, post, vectors, most, hold = re.search(r"ILi(\d)ELb\dELb(\d)ELb\dELi(n?\d+)ELi(\d+)EL\S*HoldE(\d)E", name).groups()
        if post == "0" or hold == "2" or vectors == "0" or vectors.startswith("n"):
            continue
        seen += 1
        assert int(re.search(r"\.amdhsa_group_segment_fixed_size (\d+)", meta).group(1)) <= int(most) * int(vectors) * (4 if dtype == "0" else 8) * 4 + 1024, name
    assert seen >= 12
