"""No vector or memory instruction of the built kernels comes too soon behind the matrix instruction whose result it takes.

The compiler puts idle states in between, but not in front of inline assembly, whose operands it does not look at.  Here the library's own machine code is
read: along every path from a 32x32x16 or 16x16x32 product of fp16 numbers to the first such instruction that touches its result there are as many
states as the compiler keeps between the two where it sees both.  No GPU is needed."""
import re
import struct
import subprocess

import pytest

from paper_2511_10645_amd import binding as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
STATES = {"v_mfma_f32_32x32x16_f16": 12, "v_mfma_f32_16x16x32_f16": 8}      # 8 and 4 passes of 4 cycles


def code_objects(path):
    """The gfx950 code objects that are bundled in a library."""
    data, at, magic = open(path, "rb").read(), 0, b"__CLANG_OFFLOAD_BUNDLE__"
    while (at := data.find(magic, at)) >= 0:
        n, p = struct.unpack_from("<Q", data, at + len(magic))[0], at + len(magic) + 8
        for _ in range(n):
            off, size, name = struct.unpack_from("<QQQ", data, p)
            if size and b"gfx950" in data[p + 24:p + 24 + name]:
                yield data[at + off:at + off + size]
            p += 24 + name
        at += len(magic)


def registers(text):
    """The vector registers that an operand list names."""
    out = set()
    for kind, one, lo, hi in re.findall(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        out.update((kind, i) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),)))
    return out


def kernels(listing):
    """{name: [(address, instruction, operands, target or None)]} of a disassembly."""
    out, body = {}, None
    for line in listing.splitlines():
        if m := re.match(r"^([0-9a-f]+) <(\w+)>:$", line):
            base, body = int(m[1], 16), out.setdefault(m[2], [])
        elif body is not None and (m := re.match(r"^\t(\w+)(.*?)\s*// ([0-9A-F]+):", line)):
            to = re.search(r"<\w+\+0x([0-9a-f]+)>\s*$", line) if "branch" in m[1] else None
            body.append((int(m[3], 16), m[1], m[2], base + int(to[1], 16) if to else None))
    return out


def too_soon(code, states=STATES):
    """[(address, instruction, states)] of instructions that come sooner than that behind the product whose result they touch."""
    at = {a: i for i, (a, *_) in enumerate(code)}
    leaders = sorted({0} | {at[t] for *_, t in code if t is not None} | {i + 1 for i, (_, op, *_) in enumerate(code) if "branch" in op or op == "s_endpgm"})
    leaders = [x for x in leaders if x < len(code)]
    ends = dict(zip(leaders, leaders[1:] + [len(code)]))
    needs = [registers(ops) if op.startswith(("v_", "ds_", "buffer_", "global_", "scratch_")) else None for _, op, ops, _ in code]
    found, before, work = {}, {0: {}}, [0]
    while work:
        start = work.pop()
        age = dict(before[start])                # register -> states that are still missing
        for i in range(start, ends[start]):
            _, op, ops, _ = code[i]
            if needs[i] and not op.startswith("v_mfma"):
                if late := [age[r] for r in needs[i] if r in age]:
                    found[i] = max(late + [found.get(i, 0)])
                    for r in needs[i]:
                        age.pop(r, None)
            passed = int(ops.strip()) + 1 if op == "s_nop" else 1
            age = {r: n - passed for r, n in age.items() if n > passed}
            if op.startswith("v_mfma"):
                for r in registers(ops.split(",")[0]):
                    age.pop(r, None)
                    if op in states:
                        age[r] = states[op]
        i = ends[start] - 1
        _, op, _, to = code[i]
        following = [] if op in ("s_endpgm", "s_branch") else [i + 1]
        for n in following + ([at[to]] if to is not None else []):
            if n >= len(code):
                continue
            old = before.get(n)
            new = age if old is None else {r: max(old.get(r, 0), age.get(r, 0)) for r in old.keys() | age.keys()}
            if new != old:
                before[n] = new
                work.append(n)
    return [(hex(code[i][0]), code[i][1] + code[i][2], missing) for i, missing in sorted(found.items())]


def listings(tmp_path):
    for i, code in enumerate(code_objects(B.lib_path())):
        path = tmp_path / f"{i}.elf"
        path.write_bytes(code)
        r = subprocess.run([OBJDUMP, "-d", str(path)], stdout=subprocess.PIPE, text=True, check=True)
        if any(op in r.stdout for op in STATES):
            yield r.stdout


def test_paths_are_followed():
    """The reader itself: a product's result behind a loop's branch, with and without idle states."""
    code = [(0, "v_mfma_f32_16x16x32_f16", " v[0:3], v[8:11], v[12:15], 0", None), (8, "s_cbranch_scc1", " 2", 20), (12, "s_nop", " 6", None),
            (16, "v_add_f32_e32", " v4, v4, v3", None), (20, "v_max3_f32", " v5, v0, v6, v7", None), (28, "s_endpgm", "", None)]
    assert [x[2] for x in too_soon(code)] == [7]                        # of eight, the branch is one
    code[2] = (12, "s_nop", " 5", None)
    assert [x[2] for x in too_soon(code)] == [1, 7]
    code[1] = (8, "s_nop", " 7", None)
    assert too_soon(code) == []


def test_results_are_waited_for(tmp_path):
    lists = list(listings(tmp_path))
    names = [n for text in lists for n, code in kernels(text).items() if any("mfma" in op for _, op, *_ in code)]
    assert sum("prompt_attention_kernel" in n for n in names) == 36 and sum("paged_attention_kernel" in n for n in names) == 18
    late = [(n, *x) for text in lists for n, code in kernels(text).items() for x in too_soon(code)]
    assert not late, "\n".join(map(str, late))
