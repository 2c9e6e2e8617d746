"""What a wave has stored into LDS, or is loading into it, has landed before it
reaches a workgroup barrier: read from the machine code of the built library,
on every path through every kernel.  (A barrier whose wait is missing on one
path gives right results almost always, so no run of the kernels shows it.)"""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2609_31938_amd import c3c

LLVM = "/opt/rocm/llvm/bin"


def tool(name):
    p = os.path.join(LLVM, name)
    return p if os.path.exists(p) else shutil.which(name)


pytestmark = pytest.mark.skipif(not (tool("llvm-objcopy") and tool("llvm-objdump")), reason="no LLVM binary tools")

FAR = 1 << 20  # a count of operations since an event that no path has seen


def code_objects(tmp):
    """The gfx950 code objects that the library carries, as files."""
    fat = os.path.join(tmp, "fat")
    subprocess.check_call([tool("llvm-objcopy"), f"--dump-section=.hip_fatbin={fat}", c3c.LIB_PATH, os.path.join(tmp, "copy")])
    data, out, at = open(fat, "rb").read(), [], 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(count):
            offset, size, n = struct.unpack_from("<QQQ", data, p)
            name = data[p + 24:p + 24 + n]
            p += 24 + n
            if b"gfx950" in name and size:
                out.append(os.path.join(tmp, f"code{len(out)}"))
                open(out[-1], "wb").write(data[at + offset:at + offset + size])
        at += 24
    return out


def kernels(path):
    """{name: [(address, instruction, branch target or None)]}"""
    text = subprocess.run([tool("llvm-objdump"), "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout
    out, name, base = {}, None, 0
    for line in text.splitlines():
        m = re.match(r"^([0-9a-f]+) <(\S+)>:$", line)
        if m:
            name, base = m.group(2), int(m.group(1), 16)
            out[name] = []
            continue
        m = re.match(r"^\s+(\S.*?)\s*// ([0-9A-F]+):(.*)$", line)
        if not m or name is None:
            continue
        to = None
        if m.group(1).startswith(("s_cbranch", "s_branch")):
            to = base + int(re.search(r"\+0x([0-9a-f]+)>", m.group(3)).group(1), 16) if "+0x" in m.group(3) else base
        out[name].append((int(m.group(2), 16), m.group(1), to))
    return out


def advance(ins, state, seen):
    """One instruction.  state: LDS and scalar-memory operations since the last
    LDS store that was not waited for, vector-memory operations since the last
    load into LDS that was not.  Scalar loads return out of order: they never
    count, so that only a wait for all of them serves."""
    store, load = state
    op = ins.split()[0]
    if op.startswith("ds_"):
        store = 0 if not op.startswith(("ds_read", "ds_bpermute", "ds_permute", "ds_swizzle")) else min(store + 1, FAR)
    elif op.startswith(("buffer_", "global_", "scratch_", "flat_")):
        load = 0 if "load" in op and re.search(r"_lds|\blds\b", ins) else min(load + 1, FAR)
    elif op == "s_waitcnt":
        vm, lgkm = re.search(r"vmcnt\((\d+)\)", ins), re.search(r"lgkmcnt\((\d+)\)", ins)
        if lgkm and int(lgkm.group(1)) <= store:
            store = FAR
        if vm and int(vm.group(1)) <= load:
            load = FAR
    elif op == "s_barrier":
        if store < FAR:
            seen.add("store")
        if load < FAR:
            seen.add("load")
    return store, load


def pending_at_barriers(code):
    """Whether "store"s or "load"s may be on their way at some barrier."""
    if not any(i == "s_barrier" for _, i, _ in code):
        return None
    starts = {code[0][0]} | {t for _, _, t in code if t is not None}
    blocks, cur = {}, None
    for n, (at, ins, to) in enumerate(code):
        if cur is None or at in starts:
            cur = at
            blocks[cur] = ([], [])
            if n:
                prev, last, _ = code[n - 1]
                if not last.startswith(("s_branch", "s_endpgm", "s_setpc")):
                    blocks[owner][1].append(cur)
        owner = cur
        blocks[cur][0].append(ins)
        if to is not None:
            blocks[cur][1].append(to)
        if ins.startswith(("s_cbranch", "s_branch", "s_endpgm", "s_setpc")):
            cur = None
    first, seen = code[0][0], set()
    entry, work = {first: (FAR, FAR)}, [first]
    while work:
        b = work.pop()
        state = entry[b]
        for ins in blocks[b][0]:
            state = advance(ins, state, seen)
        for s in blocks[b][1]:
            new = tuple(map(min, state, entry.get(s, (FAR + 1, FAR + 1))))
            if new != entry.get(s):
                entry[s] = new
                work.append(s)
    return seen


@pytest.fixture(scope="module")
def found(tmp_path_factory):
    out = {}
    for path in code_objects(str(tmp_path_factory.mktemp("code"))):
        for name, code in kernels(path).items():
            pending = pending_at_barriers(code) if code else None
            if pending is not None:
                out[name] = pending
    assert len(out) > 50
    return out


def test_lds_stores_have_landed(found):
    bad = [n for n, p in found.items() if "store" in p]
    assert not bad, (len(bad), bad[:4])


def test_loads_into_lds_have_landed_in_attention(found):
    """attend_many's tiles are read by all waves after a plain barrier.  (The
    kernels that count their loads, with stages still on their way at a
    barrier, wait for the one that is read next.)"""
    many = {n: p for n, p in found.items() if "attend_many" in n}
    assert many
    bad = [n for n, p in many.items() if "load" in p]
    assert not bad, (len(bad), bad[:4])


def test_the_reading_finds_a_missing_wait():
    """A loop whose store at the end meets the barrier at its head."""
    loop = [(0, "s_waitcnt lgkmcnt(0)", None), (4, "s_barrier", None), (8, "ds_write_b32 v0, v1", None),
            (12, "s_cbranch_scc1 65533", 4), (16, "s_endpgm", None)]
    assert pending_at_barriers(loop) == {"store"}
    assert pending_at_barriers(loop[:3] + [(12, "s_cbranch_scc1 65532", 0), loop[4]]) == set()
    load = [(0, "global_load_lds_dwordx4 v[0:1], off", None), (4, "global_load_dword v2, v[0:1], off", None),
            (8, "s_waitcnt vmcnt(1)", None), (12, "s_barrier", None), (16, "s_endpgm", None)]
    assert pending_at_barriers(load) == set()
    assert pending_at_barriers(load[:2] + [(8, "s_waitcnt vmcnt(2)", None)] + load[3:]) == {"load"}
