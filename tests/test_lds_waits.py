"""No kernel passes a barrier with LDS writes of its own under way.

A barrier hands LDS contents from one wave to the others, and only a wait on the
LDS counter (lgkmcnt) before it says that they have arrived.  The compiler puts
that wait before its own barriers, not before those that are written as
instructions.  The device code of the built libraries is followed here, over
all its branches, from every LDS write to the barriers that can come next.
"""

import os
import re
import shutil
import struct
import subprocess

import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                   "paper_2606_09061_amd")
OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin:" + os.environ.get("PATH", ""))
LIBS = ["libcpattn.so", "libcptree.so", "libcplayer.so", "libcppeaks.so"]


def code_objects(path):
    """The device code of a library, one object per source."""
    with open(path, "rb") as f:
        data = f.read()
    at = 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        p = at + 32
        for _ in range(struct.unpack_from("<Q", data, at + 24)[0]):
            off, size, name = struct.unpack_from("<QQQ", data, p)
            p += 24 + name
            if size:
                yield data[at + off:at + off + size]
        at += 24


def functions(listing):
    """(name, [(address, mnemonic, operands, address of the branch's target)])."""
    name, body = None, []
    for line in listing.splitlines():
        m = re.match(r"[0-9a-f]+ <(.+)>:$", line)
        if m:
            if name:
                yield name, body
            name, body = m.group(1), []
            continue
        m = re.match(r"\s+(\w+)\s*(.*?)\s*// ([0-9A-F]+): [0-9A-F ]+(?:<.*\+0x([0-9a-f]+)>|<.*>)?$",
                     line)
        if m:
            base = body[0][0] if body else int(m.group(3), 16)
            target = base + int(m.group(4) or "0", 16) if "branch" in m.group(1) else None
            body.append((int(m.group(3), 16), m.group(1), m.group(2), target))
    if name:
        yield name, body


def is_lds_write(op):
    return op.startswith("ds_") and not re.match(r"ds_(read|bpermute|permute|swizzle|nop)", op)


def waits_for_lds(op, args):
    if op != "s_waitcnt":
        return False
    m = re.search(r"lgkmcnt\((\d+)\)", args)
    return m is not None and m.group(1) == "0" or args.strip() == "0"


def barriers_with_writes(body):
    """Addresses of the barriers that a wave can reach with an LDS write behind
    it and no wait for it in between."""
    index = {addr: i for i, (addr, *_) in enumerate(body)}
    todo = [i + 1 for i, (_, op, *_) in enumerate(body) if is_lds_write(op)]
    seen, bad = set(), []
    while todo:
        i = todo.pop()
        if i in seen or i >= len(body):
            continue
        seen.add(i)
        addr, op, args, target = body[i]
        if waits_for_lds(op, args) or op == "s_endpgm":
            continue
        if op == "s_barrier":
            bad.append(hex(addr))
            continue
        assert not op.startswith(("s_setpc", "s_swappc", "s_call")), op
        if target is not None:
            todo.append(index[target])
        if op != "s_branch":
            todo.append(i + 1)
    return bad


@pytest.mark.skipif(OBJDUMP is None, reason="needs llvm-objdump")
@pytest.mark.parametrize("lib", LIBS)
def test_barriers_wait_for_lds_writes(lib, tmp_path):
    path = os.path.join(PKG, lib)
    if not os.path.exists(path):
        pytest.skip(f"{lib} is not built")
    kernels, barriers, bad = 0, 0, {}
    for n, obj in enumerate(code_objects(path)):
        f = tmp_path / f"{n}.co"
        f.write_bytes(obj)
        text = subprocess.run([OBJDUMP, "-d", str(f)], capture_output=True, text=True, check=True,
                              timeout=120).stdout
        for name, body in functions(text):
            kernels += 1
            barriers += sum(op == "s_barrier" for _, op, *_ in body)
            found = barriers_with_writes(body)
            if found:
                bad[name] = found
    assert kernels > 0 and (barriers > 0 or lib == "libcppeaks.so")
    assert not bad, bad


def test_the_walk_itself():
    """On listings written by hand: a loop, a branch around the wait, an atomic."""
    def listing(*ops):
        """One instruction every four bytes; "op args -> n" branches to the n-th."""
        out = ["0000000000000100 <k>:"]
        for i, x in enumerate(ops):
            x, _, to = x.partition(" -> ")
            out.append(f"\t{x:<40}// {0x100 + 4 * i:012X}: BF800000"
                       + (f" <k+0x{4 * int(to):x}>" if to else ""))
        return list(functions("\n".join(out)))[0][1]

    write, wait, barrier, end = ("ds_write_b128 v0, v[2:5]", "s_waitcnt lgkmcnt(0)", "s_barrier",
                                 "s_endpgm")
    assert barriers_with_writes(listing(write, wait, barrier, end)) == []
    assert barriers_with_writes(listing(write, "s_waitcnt vmcnt(0)", barrier, end)) == ["0x108"]
    assert barriers_with_writes(listing(write, "s_waitcnt lgkmcnt(1)", barrier, end)) == ["0x108"]
    assert barriers_with_writes(listing(write, "s_waitcnt vmcnt(3) lgkmcnt(0)", barrier, end)) == []
    assert barriers_with_writes(listing("ds_read_b128 v[2:5], v0", barrier, end)) == []
    assert barriers_with_writes(listing("ds_or_b64 v0, v[2:3]", barrier, end)) == ["0x104"]
    # the wait is branched around, the barrier is reached over a loop's edge
    assert barriers_with_writes(listing(write, "s_cbranch_scc0 1 -> 3", wait, barrier, end)) \
        == ["0x10c"]
    assert barriers_with_writes(listing(barrier, write, "s_cbranch_scc1 1 -> 0", end)) == ["0x100"]
    assert barriers_with_writes(listing(write, "s_branch 1 -> 3", barrier, end)) == []
