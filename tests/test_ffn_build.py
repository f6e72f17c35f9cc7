"""What the library holds of the feed-forward sublayer, without a GPU."""
import re
import shutil
import subprocess

import pytest

import paper_2602_21466_amd as lib


def _symbols(*options):
    if shutil.which("nm") is None:
        pytest.skip("no nm")
    return subprocess.run(["nm", *options, lib._build.LIB], capture_output=True, text=True, check=True).stdout


def test_kernels_for_few_rows_are_those_a_call_can_reach():
    """By the rule of few_product(): weight rows a work-group from the rows of x, the weight rows and the type."""
    want = set()
    for dtype in ("f", "DF16b", "DF16_"):
        for gate in (0, 1):
            for rows in (1, 16, 17, 32, 33, 64):
                for n in (8, 16 * 192 - 1, 16 * 192, 32 * 512 - 1, 32 * 512, 1 << 20):
                    nr = 8 if (rows <= 16 and dtype != "f") or n < 16 * 192 else 32 if gate and rows > 16 and n >= 32 * 512 else 16
                    want.add((dtype, 1 if rows <= 16 else 2 if rows <= 32 else 4, nr, gate))
    found = re.findall(r"10few_kernelI(f|DF16b|DF16_)Li(\d+)ELi(\d+)ELi(\d+)EE", _symbols("-D"))
    assert {(t, int(mt), int(nr), int(epi)) for t, mt, nr, epi in found} == want


def test_no_launcher_of_the_sublayer_is_weak():
    """A library built without one of its kernel files has to fail to load, not call a null pointer."""
    kinds = {m.group(2): m.group(1) for m in re.finditer(r"^\s*[0-9a-f]* (\w) (ffn::\w+)\(", _symbols("-DC"), re.M)}
    launchers = {k: v for k, v in kinds.items() if "launch_" in k or k == "ffn::norm_workspace_floats"}
    assert {"ffn::launch_tile_fp32", "ffn::launch_few_grad", "ffn::norm_workspace_floats"} <= set(launchers)
    assert set(launchers.values()) == {"T"}, launchers
