"""Registers of the library's kernels that are held in scratch memory, read from the library without a GPU."""
import struct

import paper_2602_21466_amd as lib


def _kernels():
    """{kernel's name: bytes of scratch a lane} of every gfx950 code object in the library."""
    data = open(lib._build.LIB, "rb").read()
    magic, found, at = b"__CLANG_OFFLOAD_BUNDLE__", {}, 0
    while (at := data.find(magic, at)) >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count):
            offset, size, n = struct.unpack_from("<3Q", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + n]:
                found.update(_descriptors(data[at + offset:at + offset + size]))
            entry += 24 + n
        at += len(magic)
    return found


def _descriptors(elf):
    """Of an ELF file's symbols NAME.kd, kernel descriptors: their second word is the scratch a lane."""
    assert elf[:5] == b"\x7fELF\x02"
    start, = struct.unpack_from("<Q", elf, 40)
    size, count = struct.unpack_from("<2H", elf, 58)
    sections = [struct.unpack_from("<2I4Q2I2Q", elf, start + i * size) for i in range(count)]
    out = {}
    for _, kind, _, _, offset, length, link, _, _, each in sections:
        if kind != 11:   # the dynamic symbols
            continue
        names = sections[link][4]
        for i in range(offset, offset + length, each):
            name, _, _, section, value, _ = struct.unpack_from("<I2BH2Q", elf, i)
            name = elf[names + name:elf.index(b"\0", names + name)].decode()
            if name.endswith(".kd"):
                _, _, _, address, where, *_ = sections[section]
                out[name[:-3]] = struct.unpack_from("<2I", elf, where + value - address)[1]
    return out


def test_layer_norm_and_mixtures_hold_their_values_in_registers():
    kernels = _kernels()
    kinds = ("layer_forward_kernel", "layer_means_kernel", "layer_columns_kernel", "layer_forward_rows", "layer_backward_rows",
             "sort_count_kernel", "sort_place_kernel", "gather_kernel", "combine_kernel", "combine_parts_kernel",
             "combine_backward_kernel", "expert_rows_kernel", "expert_rows_deep_kernel", "expert_grads_kernel",
             "expert_few_kernel", "join_sums_kernel")
    for kind in kinds:
        some = {k: v for k, v in kernels.items() if kind in k}
        assert some, kind
        assert not any(some.values()), {k: v for k, v in some.items() if v}
