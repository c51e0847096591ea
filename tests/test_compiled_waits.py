"""The listing of the library's kernels as they were built: no instruction reads or overwrites the registers of a matrix product before it has left them there.

The matrix unit writes its result some cycles after it was started, and other units do not wait for it: that many instructions, or s_nop, have to lie between, on
every path.  The compiler sees to that, but once did not, behind a loop; results were wrong in two registers of sixteen.  A product of n passes of four cycles asks
for n + 3 (fp32 operands: n + 1; n from the instruction's size) before a vector, memory or LDS instruction that names one of its registers."""
import os
import re
import subprocess

import pytest

from paper_2309_03523_amd import binding

LLVM = "/opt/rocm/llvm/bin/"
WAIT = {"32x32x16_bf16": 11, "32x32x8_bf16_1k": 11, "32x32x16_f16": 11, "16x16x32_bf16": 7, "16x16x16_bf16": 7, "16x16x16_bf16_1k": 7, "16x16x32_f16": 7, "16x16x4_f32": 9,
        "32x32x2_f32": 17}
OTHERS = re.compile(r"v_|ds_|global_|buffer_|scratch_|flat_")


def _registers(text):
    """The vector registers that operands name."""
    out = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out.update(kind + str(i) for i in range(int(a), int(b) + 1))
    out.update(kind + i for kind, i in re.findall(r"\b([va])(\d+)\b", text))
    return out


def _too_early(code):
    """code: [(opcode, operands, index of the branch target or None)].  Pairs (product, reader) that lie too near."""
    found = []
    for i, (op, args, _) in enumerate(code):
        if not op.startswith("v_mfma_f32_") or op[11:] not in WAIT:
            continue
        need, dst = WAIT[op[11:]], _registers(args.split(",")[0])
        todo, seen = [(i + 1, 0)], {}
        while todo:
            j, waited = todo.pop()
            if j >= len(code) or waited >= need or seen.get(j, need) <= waited:
                continue
            seen[j] = waited
            o, a, target = code[j]
            if o == "s_endpgm":
                continue
            if o.startswith("v_mfma"):
                if _registers(a.split(",")[0]) & dst:       # a chain of products waits by itself
                    continue
            elif OTHERS.match(o) and _registers(a) & dst:
                found.append((i, j, waited, need))
                continue
            if target is not None:
                todo.append((target, waited + 1))
            if o != "s_branch":
                todo.append((j + 1, waited + (int(a.split()[0], 0) + 1 if o == "s_nop" else 1)))
    return found


def _kernels(listing):
    """(name, code) of each function of a listing."""
    name, lines = None, []
    for line in listing:
        m = re.match(r"^([0-9a-f]+) <(.+)>:", line)
        if m:
            if name:
                yield name, lines
            name, lines = m.group(2), []
        elif "//" in line:
            lines.append(line)
    if name:
        yield name, lines


def _parsed(name, lines):
    at, code = {}, []
    for line in lines:
        text, _, note = line.partition("//")
        place = int(note.split(":")[0], 16)
        at[place] = len(code)
        op, _, args = text.strip().partition(" ")
        target = re.search(r"<[^>]*?(?:\+0x([0-9a-f]+))?>\s*$", note) if op.startswith(("s_branch", "s_cbranch")) else None
        code.append([op, args.strip(), int(target.group(1) or "0", 16) if target else None])
    first = min(at) if at else 0
    for c in code:
        if c[2] is not None:
            c[2] = at[first + c[2]]
    return code


def test_the_search_finds_what_it_looks_for():
    """In small listings: a reader behind the loop that the product ends, and the same with enough in between."""
    product = ("v_mfma_f32_32x32x16_bf16", "v[18:33], v[8:11], v[66:69], v[18:33]", None)
    reader = ("v_mov_b64_e32", "v[96:97], v[32:33]", None)
    loop = [product, ("s_cbranch_vccnz", "0", 3), ("s_branch", "0", 0), reader, ("s_endpgm", "", None)]
    assert _too_early(loop) == [(0, 3, 1, 11)]
    assert _too_early([product, ("s_nop", "7", None), ("s_nop", "2", None), reader, ("s_endpgm", "", None)]) == []
    assert _too_early([product, ("s_nop", "7", None), ("s_nop", "1", None), reader, ("s_endpgm", "", None)]) == [(0, 3, 10, 11)]
    assert _too_early([product, ("v_mov_b32_e32", "v34, v17", None), product, ("s_endpgm", "", None)]) == []


def test_every_kernel_waits_for_its_products(tmp_path):
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    if not all(os.path.exists(LLVM + t) for t in ("llvm-objcopy", "llvm-objdump")):
        pytest.skip("no disassembler")
    fat = tmp_path / "fat.bin"
    subprocess.run([LLVM + "llvm-objcopy", "-O", "binary", "--only-section=.hip_fatbin", binding.LIB_PATH, str(fat)], check=True)
    image = fat.read_bytes()
    starts = [m.start() for m in re.finditer(b"\x7fELF\x02", image)] + [len(image)]
    products = 0
    for k, (a, b) in enumerate(zip(starts, starts[1:])):
        part = tmp_path / f"code{k}.o"
        part.write_bytes(image[a:b])
        listing = subprocess.run([LLVM + "llvm-objdump", "-d", "--mcpu=gfx950", str(part)], check=True, capture_output=True, text=True).stdout
        part.unlink()
        if "v_mfma" not in listing:
            continue
        for name, lines in _kernels(listing.splitlines()):
            if not any("v_mfma_f32" in line for line in lines):
                continue
            code = _parsed(name, lines)
            kinds = [op[11:] for op, *_ in code if op.startswith("v_mfma_f32_")]
            assert not set(kinds) - set(WAIT), f"{name}: products that this test does not know"
            products += len(kinds)
            early = _too_early(code)
            assert not early, f"{name}: " + "; ".join(f"{code[i][0]} {code[i][1]} and {code[j][0]} {code[j][1]} {w} of {n} apart" for i, j, w, n in early[:3])
    assert products > 1000
