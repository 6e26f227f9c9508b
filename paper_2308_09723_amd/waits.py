"""Waits between matrix products and what reads their results, looked for in the objects that the compiler made.

gfx950 does not hold a vector instruction back until a matrix product that it depends on has written its registers: so many wait states have to lie between them (a product of
2 passes: 5, of 4: 8, of 8: 12; a pass is four cycles, as is a state: an instruction, or each of s_nop's), and the compiler puts them there.  Where several ways lead to an
instruction this one was seen to count along a longer one: a sum in an accumulation register was read one state behind a loop's last product, and a result was wrong; scores that a
branch leads past the search for their maximum were read 10 or 11 states behind instead of 12.  short_waits() follows every way.
"""
from __future__ import annotations

import re

# By shape; all that the kernels use is here
PASSES = {"4x4x4": 2, "16x16x32": 4, "16x16x64": 4, "32x32x16": 8}

_REGISTERS = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")
_STORES = re.compile(r"(ds_write|ds_store|ds_bpermute|ds_permute|(global|buffer|flat|scratch)_(store|atomic))")


def needed(product: str) -> int:
    """Wait states behind a product (a KeyError for one that PASSES does not know)."""
    passes = PASSES[re.search(r"_(\d+x\d+x\d+)", product).group(1)]
    return passes + 3 + (passes > 2)


def _registers(operands):
    out = set()
    for kind, first, last, one in _REGISTERS.findall(operands):
        out |= {(kind, i) for i in (range(int(first), int(last) + 1) if first else (int(one),))}
    return out


def _kernels(assembly):
    """(name, [(mnemonic, operands)]) of each function of llvm-objdump's output; labels are (":", name)."""
    name, lines = None, []
    for line in assembly.splitlines():
        line = line.split("//")[0].strip()
        m = re.match(r"<(.+)>:$", line)
        if m and re.fullmatch(r"L\d+", m.group(1)):
            lines.append((":", m.group(1)))
        elif m:
            if name:
                yield name, lines
            name, lines = m.group(1), []
        elif name and re.match(r"[a-z]\w*( |$)", line):
            mnemonic, _, operands = line.partition(" ")
            lines.append((mnemonic, operands.strip()))
    if name:
        yield name, lines


def short_waits(assembly: str):
    """[(kernel, product, instruction, states, needed)]: for each product the first instruction found that uses its result too early."""
    found = []
    for name, lines in _kernels(assembly):
        labels = {operands: i for i, (mnemonic, operands) in enumerate(lines) if mnemonic == ":"}
        for start, (product, operands) in enumerate(lines):
            if not product.startswith(("v_mfma", "v_smfmac")):
                continue
            need = needed(product)
            ways, least, early = [(start + 1, 0, frozenset(_registers(operands.split(", ")[0])))], {}, None
            while ways and not early:
                at, states, result = ways.pop()
                if at >= len(lines) or states >= need or not result or least.get((at, result), need) <= states:
                    continue
                least[at, result] = states
                mnemonic, rest = lines[at]
                if mnemonic == ":":
                    ways.append((at + 1, states, result))
                elif mnemonic == "s_nop":
                    ways.append((at + 1, states + int(rest, 0) + 1, result))
                elif mnemonic == "s_branch":
                    ways.append((labels[rest], states + 1, result))
                elif mnemonic.startswith("s_cbranch"):
                    ways += [(labels[rest], states + 1, result), (at + 1, states + 1, result)]
                elif mnemonic == "s_endpgm":
                    pass
                elif mnemonic.startswith("s_"):
                    ways.append((at + 1, states + 1, result))
                else:
                    parts = rest.split(", ")
                    matrix, stores = mnemonic.startswith(("v_mfma", "v_smfmac")), _STORES.match(mnemonic)
                    # (a product may add to what the one before it wrote: the hardware passes that on)
                    read = _registers(", ".join(parts if stores else parts[1:3] if matrix else parts[1:]))
                    written = set() if stores else _registers(parts[0])
                    if read & result or (written & result and not matrix):
                        early = (name, f"{product} {operands}", f"{mnemonic} {rest}", states, need)
                    else:
                        ways.append((at + 1, states + 1, result - written))
            if early:
                found.append(early)
    return found
