"""What the library holds of the experts' operators and of the layer norm, without a GPU."""
import re

import paper_2602_21466_amd as lib
from test_ffn_build import _symbols


def test_kernels_for_few_rows_are_those_a_call_can_reach():
    """By the rules of few_rows() and few_cut(): rows a tile from the mean of an expert's rows, weight rows a work-group from
    all experts' of a product, the rows a tile and the type."""
    want = set()
    for dtype in ("f", "DF16b", "DF16_"):
        wide = dtype == "f"
        for gate in (0, 1):
            for mean in range(1, 29 if wide else 49):
                for n in (8, 16 * 200 - 1, 16 * 200, 32 * 256 - 1, 32 * 256, 1 << 20):
                    rows = 16 if mean <= (10 if wide else 6) else 32 if mean <= 24 or wide else 64
                    nr = 32 if n >= 32 * 256 and rows > 16 else 16
                    if n < 16 * 200 or (gate and rows == 16 and not wide):
                        nr = 8
                    want.add((dtype, rows // 16, nr, gate))
    found = re.findall(r"17expert_few_kernelI(f|DF16b|DF16_)Li(\d+)ELi(\d+)ELi(\d+)EE", _symbols("-D"))
    assert {(t, int(mt), int(nr), int(epi)) for t, mt, nr, epi in found} == want


def test_tiles_of_the_experts_products():
    """Both tile widths of the forward products (results, hidden rows, sums in parts) and of the hidden rows' gradient, three
    steps in flight for 128-wide tiles of 16-bit arrays alone, and the gradients' products."""
    rows = [(bc, epi) for bc, epis in ((0, (0, 1, 3)), (1, (2, 3))) for epi in epis]
    names = _symbols("-D")
    found = set(re.findall(r"18expert_rows_kernelI(f|DF16b|DF16_)Li(\d+)ELb([01])ELi(\d)EE", names))
    assert found == {(t, tile, str(bc), str(epi)) for t in ("f", "DF16b", "DF16_") for tile in ("128", "256") for bc, epi in rows}
    found = set(re.findall(r"23expert_rows_deep_kernelI(f|DF16b|DF16_)Lb([01])ELi(\d)EE", names))
    assert found == {(t, str(bc), str(epi)) for t in ("DF16b", "DF16_") for bc, epi in rows}
    found = set(re.findall(r"19expert_grads_kernelI(f|DF16b|DF16_)Li(\d+)EE", names))
    assert found == {(t, tile) for t in ("f", "DF16b", "DF16_") for tile in ("128", "256")}


def test_no_launcher_is_weak():
    """A library built without one of its kernel files has to fail to load, not call a null pointer."""
    kinds = {m.group(2): m.group(1) for m in re.finditer(r"^\s*[0-9a-f]* (\w) (ffn::\w+)\(", _symbols("-DC"), re.M)}
    names = {"ffn::launch_%s_%s" % (n, t) for n in ("expert_rows", "expert_few", "expert_grads", "layer_forward", "layer_backward")
             for t in ("fp32", "bf16", "fp16")}
    names |= {"ffn::launch_" + n for n in ("sort", "gather", "combine", "combine_parts", "combine_backward", "join_sums")}
    names.add("ffn::layer_workspace_floats")
    assert names <= set(kinds) and {kinds[n] for n in names} == {"T"}


def test_each_name_of_the_header_is_exported():
    exported = set(lib.exported_symbols())
    for n in ("ffn_route", "ffn_route_workspace_bytes", "ffn_route_gather", "ffn_route_combine", "ffn_route_combine_backward",
              "ffn_experts_plan", "ffn_experts_destroy", "ffn_experts_workspace_bytes", "ffn_experts_backward_workspace_bytes",
              "ffn_experts_forward", "ffn_experts_backward", "ffn_layer_forward", "ffn_layer_backward", "ffn_layer_workspace_bytes"):
        assert n in exported and callable(getattr(lib, n))
