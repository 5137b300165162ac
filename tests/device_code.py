"""The library's own kernels as the compiler left them: instructions and the ways through them (no GPU needed)."""
import os
import re
import shutil
import subprocess

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# "	s_cbranch_scc1 12     // 0000000023AC: BF85000C <symbol+0x1234>"
LINE = re.compile(r"^\s+(\S+)(.*?)\s*//\s*([0-9A-F]+):[^<]*(?:<[^+>]*(?:\+0x([0-9a-f]+))?>)?\s*$")


def available():
    return os.path.exists(OBJDUMP)


def kernels(library, folder, what):
    """{name: [(address, opcode, operands, address it may jump to or None), ..]} of the kernels whose mangled name has `what`."""
    copy = os.path.join(str(folder), "library.so")
    shutil.copy(library, copy)
    subprocess.run([OBJDUMP, "--offloading", copy], check=True, capture_output=True, cwd=str(folder))
    out = {}
    for name in sorted(os.listdir(str(folder))):
        path = os.path.join(str(folder), name)
        if "gfx950" not in name or what.encode() not in open(path, "rb").read():
            continue
        text = subprocess.run([OBJDUMP, "-d", path], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text)[1:]:
            head, *lines = part.splitlines()
            start, symbol = re.match(r"([0-9a-f]+) <(.*)>:", head).groups()
            if what not in symbol:
                continue
            code = []
            for line in lines:
                m = LINE.match(line)
                if m:
                    op, operands, at, jump = m.groups()
                    to = None
                    if "branch" in op:
                        assert "<" in line, line
                        to = int(start, 16) + int(jump or "0", 16)
                    code.append((int(at, 16), op, operands.strip(), to))
            out[symbol] = code
    return out


def reaching(code, step):
    """Walks every way through a kernel: `step(op, operands, state)` gives the truth value behind an instruction from that in front of it; where
    ways meet, one True is enough.  {index of an instruction: the state in front of it}."""
    index = {at: i for i, (at, *_) in enumerate(code)}
    before, todo = {0: False}, [0]
    while todo:
        i = todo.pop()
        state = before[i]
        while True:
            _, op, operands, to = code[i]
            state = step(op, operands, state)
            ways = []
            if op not in ("s_endpgm", "s_branch", "s_setpc_b64"):
                ways.append(i + 1)
            if to is not None:
                ways.append(index[to])
            ways = [w for w in ways if w < len(code) and (w not in before or (state and not before[w]))]
            for w in ways:
                before[w] = state
            if not ways:
                break
            i = ways[0]
            todo += ways[1:]
    return before
