"""Wait states between matrix products and what uses them, in the disassembly of the kernels
built here.

A v_mfma_*_16x16x32 of bf16 takes four passes: on gfx950 another instruction may use its
result eight wait states after it.  Every instruction between counts as one, s_nop n as n + 1.
The accumulator of a further product of the same kind needs none.
"""
from __future__ import annotations

import functools
import os
import re
import shutil
import struct
import subprocess

WAITS = 8
PRODUCT = re.compile(r"v_mfma_f32_16x16x32_bf16\b")
_MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
_REGS = re.compile(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])")


def objdump():
    for path in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")):
        if path and os.path.exists(path):
            return path
    return None


def code_objects(library):
    """The gfx950 code objects that a host library holds."""
    with open(library, "rb") as f:
        data = f.read()
    at = data.find(_MAGIC)
    while at >= 0:
        count, place = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            name = data[place + 24:place + 24 + length]
            place += 24 + length
            if b"gfx950" in name and size:
                yield data[at + offset:at + offset + size]
        at = data.find(_MAGIC, at + len(_MAGIC))


def disassemble(code, folder):
    path = os.path.join(folder, "code.elf")
    with open(path, "wb") as f:
        f.write(code)
    with open(path + ".txt", "wb") as f:
        subprocess.run([objdump(), "-d", "--mcpu=gfx950", path], check=True, stdout=f)
    with open(path + ".txt") as f:
        return f.read()


@functools.lru_cache(maxsize=None)
def _registers(text):
    out = set()
    for kind, one, first, last in _REGS.findall(text):
        lo, hi = (int(one), int(one)) if one else (int(first), int(last))
        out.update((kind, i) for i in range(lo, hi + 1))
    return frozenset(out)


_VECTOR = ("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")
_LINE = re.compile(r"^[ \t]+(\S+)[ \t]*(.*?)[ \t]*// ([0-9A-F]+):(.*)$", re.MULTILINE)
_HEAD = re.compile(r"([0-9a-f]+) <(.+)>:\n")


def kernels(listing):
    """(name, instructions) of the kernels with such products; an instruction is (address, operation, operands, target
    or None)."""
    for text in re.split(r"\n(?=[0-9a-f]+ <)", "\n" + listing):
        head = _HEAD.match(text)
        if not head or not PRODUCT.search(text):
            continue
        start, body = int(head.group(1), 16), []
        for op, operands, address, rest in _LINE.findall(text):
            target = None
            if op.startswith(("s_branch", "s_cbranch")):
                target = start + int(re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>", rest).group(1) or "0", 16)
            body.append((int(address, 16), op, operands, target))
        yield head.group(2), body


def early_uses(body):
    """(address of a product, address of an early use, wait states between) for all ways through a kernel."""
    index = {a: i for i, (a, _, _, _) in enumerate(body)}
    found = []
    for i, (address, op, operands, _) in enumerate(body):
        if not PRODUCT.match(op):
            continue
        result = _registers(operands.split(",")[0])
        best = {}                                     # instruction -> fewest wait states before it
        todo = [(i + 1, 0)]
        while todo:
            j, waits = todo.pop()
            if j >= len(body) or waits >= WAITS or best.get(j, WAITS) <= waits:
                continue
            best[j] = waits
            _, other, text, target = body[j]
            if other.startswith(_VECTOR) and _registers(text) & result:
                fields = [f.strip() for f in text.split(",")]
                own = PRODUCT.match(other) and not _registers(",".join(fields[1:3])) & result
                if not own:
                    found.append((address, body[j][0], waits))
                continue                              # (what follows a use waits for that, or is the accumulator's)
            waits += int(text.split()[0], 0) + 1 if other == "s_nop" else 1
            if other == "s_endpgm":
                continue
            if target is not None:
                todo.append((index[target], waits))
                if other == "s_branch":
                    continue
            todo.append((j + 1, waits))
    return found
