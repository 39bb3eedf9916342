"""Every barrier of the built library, in the AMD assembly it was compiled to: no wave reaches one with LDS operations outstanding.  (A
compiler that drops such a wait makes a race that shows now and then, by the timing of the other waves.)"""
import os
import re
import struct
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2605_05838_amd import binding

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
NEVER = 1000


def code_objects(data):
    """The gfx950 code objects of a library: of every bundle, entries of (offset, size, length of the target's name) and the name."""
    at = data.find(MAGIC)
    while at >= 0:
        n, p = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(n):
            off, size, ln = struct.unpack_from("<QQQ", data, p)
            name, p = data[p + 24:p + 24 + ln].decode(), p + 24 + ln
            if "gfx950" in name and size:
                yield data[at + off:at + off + size]
        at = data.find(MAGIC, at + 24)


def kernels(text):
    """{name: [(address, instruction)]} of a disassembly."""
    out, cur = {}, None
    for line in text.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if m:
            cur = out.setdefault(m.group(1), [])
            continue
        m = re.match(r"^\s+(\S.*?)\s*// ([0-9A-F]+):", line)
        if m and cur is not None:
            cur.append((int(m.group(2), 16), m.group(1)))
    return out


def unfinished(code):
    """[(address, what)] of the barriers that an LDS read or write may be outstanding at.  Counted in order (lgkmcnt(N): all but the last N are
    done): per place, how many operations came after the last write, and the last read, that may be outstanding; the fewest over all ways there."""
    index = {a: i for i, (a, _) in enumerate(code)}
    state = {0: (NEVER, NEVER)}
    todo, found = [0], set()
    while todo:
        i = todo.pop()
        w, r = state[i]
        while i < len(code):
            addr, s = code[i]
            op, targets = s.split()[0], []
            if op.startswith("ds_") or op.startswith(("s_load", "s_buffer_load")):
                w, r = min(w + 1, NEVER), min(r + 1, NEVER)
                if op.startswith("ds_"):
                    reads = "read" in op or "bpermute" in op or "permute" in op or "swizzle" in op
                    w, r = (w, 1) if reads else (1, r)
            elif op == "s_waitcnt":
                m = re.search(r"lgkmcnt\((\d+)\)", s)
                n = int(m.group(1)) if m else NEVER
                w, r = (NEVER if w > n else w), (NEVER if r > n else r)
            elif op == "s_barrier":
                found |= {(addr, what) for what, x in (("write", w), ("read", r)) if x < NEVER}
            m = re.match(r"s_c?branch\S*\s+(\d+)", s)
            if m:
                k = int(m.group(1))
                targets.append(index[addr + 4 + 4 * (k - 65536 if k >= 32768 else k)])
                if op != "s_branch":
                    targets.append(i + 1)
            elif op == "s_endpgm":
                break
            elif i + 1 in state or i + 1 >= len(code):
                targets.append(i + 1)
            if targets:
                for t in targets:
                    old = state.get(t, (NEVER + 1, NEVER + 1))
                    new = (min(old[0], w), min(old[1], r))
                    if new != old:
                        state[t] = new
                        todo.append(t)
                break
            i += 1
    return sorted(found)


def test_the_reading_of_a_loop():
    """A write at the end of a loop that begins with a barrier, with and without the wait; one that a later read's wait covers; one that it does not."""
    loop = lambda *body: [(4 * i, s) for i, s in enumerate(("s_nop 0", "s_barrier", *body, "s_cbranch_scc1 %d" % (65536 - 2 - len(body)), "s_endpgm"))]
    assert unfinished(loop("ds_write_b32 v0, v1")) == [(4, "write")]
    assert unfinished(loop("ds_write_b32 v0, v1", "s_waitcnt lgkmcnt(0)")) == []
    assert unfinished(loop("ds_write_b32 v0, v1", "ds_read_b32 v2, v3", "s_waitcnt lgkmcnt(1)")) == [(4, "read")]
    assert unfinished(loop("ds_read_b32 v2, v3", "ds_write_b32 v0, v1", "s_waitcnt lgkmcnt(1)")) == [(4, "write")]
    assert unfinished(loop("ds_write_b32 v0, v1", "s_waitcnt vmcnt(0) lgkmcnt(0)")) == []


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_no_barrier_meets_lds_operations(tmp_path):
    with open(binding.LIB_PATH, "rb") as f:
        data = f.read()
    paths = []
    for i, o in enumerate(code_objects(data)):
        paths.append(str(tmp_path / ("%d.co" % i)))
        with open(paths[-1], "wb") as f:
            f.write(o)
    dump = lambda p: subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", p], check=True, capture_output=True, text=True).stdout
    barriers, bad = 0, {}
    with ThreadPoolExecutor(4) as pool:
        for text in pool.map(dump, paths):
            for name, code in kernels(text).items():
                barriers += sum(s == "s_barrier" for _, s in code)
                if found := unfinished(code):
                    bad[name] = found
    assert barriers > 100, "the library's kernels were not found"
    assert not bad, (len(bad), {k: ["%x %s" % x for x in v] for k, v in list(bad.items())[:4]})
