"""What the vocabulary's kernels' code must not hold, read from the assembly that the library's compiler and flags make of their
sources; no GPU.  The library allocates nothing, so none of them keeps anything in scratch memory, which the runtime would have to allocate; and LDS is
filled only by loads that are waited for."""
import os
import re
import subprocess

import pytest

from paper_2409_02423_amd import build

SOURCES = [s for s in build.SOURCES if os.path.basename(s).startswith("ze_")]


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


@pytest.mark.parametrize("source, least", (("ze_embedding.hip", 20), ("ze_loss.hip", 40)))
def test_no_kernel_uses_scratch(assembly, source, least):
    kernels = re.findall(r"\.amdhsa_kernel (\S+)\n(.*?)\.end_amdhsa_kernel", assembly[source], flags=re.S)
    assert len(kernels) >= least
    for name, meta in kernels:
        assert re.search(r"\.amdhsa_private_segment_fixed_size (\d+)", meta).group(1) == "0", name
        assert int(re.search(r"\.amdhsa_group_segment_fixed_size (\d+)", meta).group(1)) <= 160 * 1024, name


def test_loads_into_lds_are_waited_for_before_the_end(assembly):
    """Between a kernel's last load into LDS and its end there is a wait for all loads."""
    text = assembly["ze_loss.hip"]
    seen = 0
    for name in re.findall(r"\.amdhsa_kernel (\S+)", text):
        body = re.search(r"^%s:.*?^\.Lfunc_end" % re.escape(name), text, flags=re.S | re.M).group(0)
        last = max((m.end() for m in re.finditer(r"buffer_load_dwordx4 .*lds", body)), default=None)
        if last is None:
            continue
        seen += 1
        assert re.search(r"s_waitcnt vmcnt\(0\)", body[last:]), name
    assert seen >= 30


def test_large_products_keep_their_sums_in_place(assembly):
    """Where the order of instructions is written down, a step holds its products, its reads and its loads, and moves no sum; and between a step's last product and
    the first use of a sum there are eleven issues (two s_nop), which the compiler does not see to in instructions by name."""
    text = assembly["ze_loss.hip"]
    seen = 0
    for name in re.findall(r"\.amdhsa_kernel (\S*Lb1E\S*)", text):
        if "finish" in name:
            continue
        nx, ny, stages = (int(v) for v in re.search(r"ShapeILi(\d+)ELi(\d+)ELi2ELi2ELi(\d)E", name).groups())
        body = re.search(r"^%s:.*?^\.Lfunc_end" % re.escape(name), text, flags=re.S | re.M).group(0)
        each = 2 * (nx // 32) * (ny // 32)
        steps = [b for b in re.split(r"^\.LBB\S+:", body, flags=re.M) if b.count("v_mfma") >= each]
        assert sum(b.count("v_mfma") for b in steps) >= stages * each, name
        for b in steps:
            inside = b[b.index("v_mfma"):b.rindex("v_mfma")]
            assert "v_accvgpr" not in inside and "scratch" not in inside and "v_mov_b32" not in inside, name
        waits = [m.start() for m in re.finditer(r"s_nop 7\n\ts_nop 3", body)]
        assert waits, name
        for at in waits:
            assert "v_accvgpr" not in body[body.rindex("v_mfma", 0, at):at], name
        seen += 1
    assert seen >= 14


def test_half_tiles_of_the_hidden_gradient_have_three_steps_under_way(assembly):
    """Kernels of that gradient with two, which the other products' half tiles have, would have no caller."""
    stages = {}
    for kind, n in re.findall(r"\.amdhsa_kernel \S*\d([a-z_]+_kernel)ILi\dENS_5ShapeILi256ELi128ELi2ELi2ELi(\d)E", assembly["ze_loss.hip"]):
        stages.setdefault(kind, set()).add(n)
    assert stages == {"logits_kernel": {"2"}, "gradient_kernel": {"2"}, "table_gradient_kernel": {"2"}, "hidden_gradient_kernel": {"3"}, "hidden_finish_kernel": {"3"}}
