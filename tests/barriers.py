"""What reaches the barriers of the library's kernels: the built code objects are disassembled, and every path to an s_barrier is followed with what is under way on it.  Test infrastructure.

A wave passes an s_barrier with its own LDS accesses still on their way: s_barrier waits for waves, not for memory, and what another wave then reads may not be there yet.  So an LDS write (or a load from
memory into LDS) has to be waited for, by lgkmcnt (or vmcnt), on every path between it and the barrier.  Compilers put these waits in by themselves, and have left one out at the head of a loop.
"""
import collections
import glob
import os
import re
import shutil
import subprocess
import tempfile

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LINE = re.compile(r"^\s+(\S+)(.*?)\s*//\s*([0-9A-F]+):")
TARGET = re.compile(r"<([^>+]+)(?:\+0x([0-9a-f]+))?>\s*$")
NO_MEMORY = ("ds_bpermute", "ds_permute", "ds_swizzle", "ds_nop")   # (they cross lanes, and touch no memory)
NEVER = 1 << 20


def functions(lib):
    """{kernel: [(address, mnemonic, operands, branch target or None)]} of all code objects in a shared library."""
    found = {}
    with tempfile.TemporaryDirectory(prefix="barriers_") as tmp:
        shutil.copy(lib, os.path.join(tmp, "lib.so"))
        subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp, check=True, capture_output=True)
        for obj in sorted(glob.glob(os.path.join(tmp, "lib.so.*gfx*"))):
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", obj], check=True, capture_output=True, text=True).stdout
            found.update(parse(text))
    return found


def parse(text):
    found, now, base = {}, None, 0
    for line in text.splitlines():
        head = re.match(r"^([0-9a-f]+) <(\S+)>:", line)
        if head:
            now, base = found.setdefault(head.group(2), []), int(head.group(1), 16)
            continue
        m = LINE.match(line)
        if m is None or now is None:
            continue
        op, args, at = m.group(1), m.group(2).strip(), int(m.group(3), 16)
        target = None
        if op.startswith(("s_branch", "s_cbranch")):
            t = TARGET.search(line)
            target = base + int(t.group(2) or "0", 16)
        now.append((at, op, args, target))
    return found


def counts(args):
    """(vmcnt, lgkmcnt) that an s_waitcnt waits for; NEVER: not for that one."""
    got = [NEVER, NEVER]
    for i, name in enumerate(("vmcnt", "lgkmcnt")):
        m = re.search(name + r"\((\d+)\)", args)
        if m:
            got[i] = int(m.group(1))
    if "cnt(" not in args and args:
        raw = int(args, 0)
        got = [(raw & 15) | (raw >> 10 & 48), raw >> 8 & 15]
    return got


# What is under way: the operations of its counter that were issued after the youngest LDS write, LDS read, load into LDS (None: nothing is), and whether scalar loads are (they come in any order).
State = collections.namedtuple("State", "write read direct scalar")


def step(s, op, args):
    if op == "s_waitcnt":
        vm, lgkm = counts(args)
        clear = lambda at, n: None if at is None or n <= at else at   # noqa: E731
        if s.scalar and lgkm:
            lgkm = NEVER
        return State(clear(s.write, lgkm), clear(s.read, lgkm), clear(s.direct, vm), s.scalar and lgkm != 0)
    more = lambda at: None if at is None else at + 1   # noqa: E731
    if op.startswith("ds_"):
        s = s._replace(write=more(s.write), read=more(s.read))
        if op.startswith(NO_MEMORY):
            return s
        return s._replace(read=0) if op.startswith("ds_read") else s._replace(write=0)
    if op.startswith(("s_load", "s_buffer_load", "s_scratch", "s_memtime", "s_memrealtime", "s_sendmsg", "s_getreg")):
        return s._replace(write=more(s.write), read=more(s.read), scalar=True) if not op.startswith("s_getreg") else s
    if op.startswith(("buffer_", "global_", "scratch_", "flat_")) and not op.startswith(("buffer_wbl2", "buffer_inv")):
        s = s._replace(direct=more(s.direct))
        if op.startswith("flat_"):
            s = s._replace(write=more(s.write), read=more(s.read))
        return s._replace(direct=0) if re.search(r"\blds\b", args) or "_lds_" in op else s
    return s


def join(a, b):
    least = lambda x, y: y if x is None else x if y is None else min(x, y)   # noqa: E731
    return State(least(a.write, b.write), least(a.read, b.read), least(a.direct, b.direct), a.scalar or b.scalar)


def unwaited(code):
    """Barriers that a path reaches with LDS writes or loads into LDS under way: [(address, what)]."""
    index = {at: i for i, (at, _, _, _) in enumerate(code)}
    before, todo = {0: State(None, None, None, False)}, [0]
    while todo:
        i = todo.pop()
        s = before[i]
        while True:
            at, op, args, target = code[i]
            s = step(s, op, args)
            nexts = []
            if target is not None:
                nexts.append(index[target])
            if op not in ("s_branch", "s_endpgm", "s_setpc_b64") and i + 1 < len(code):
                nexts.append(i + 1)
            changed = []
            for n in nexts:
                new = s if n not in before else join(before[n], s)
                if n not in before or new != before[n]:
                    before[n] = new
                    changed.append(n)
            if not changed:
                break
            todo += changed[1:]
            i = changed[0]
            s = before[i]
    bad = []
    for i, (at, op, _, _) in enumerate(code):
        if op == "s_barrier" and i in before:
            s = before[i]
            bad += [(at, what) for what, on in (("an LDS write", s.write), ("a load into LDS", s.direct)) if on is not None]
    return bad
