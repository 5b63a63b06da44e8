"""No wave reaches a barrier with writes into LDS of its own on their way: in the assembly that the compiler writes for
the 4-bit attention's kernels, on every path.  (A bare s_barrier waits for nothing, and what lies behind it may use the same
place in LDS.)  No GPU is involved."""
import os
import re
import subprocess

import pytest

from paper_2609_24197_amd import build

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="hipcc not installed")

READS = re.compile(r"ds_(read|bpermute|permute|swizzle)")


def functions(asm):
    """(name, instructions) of each kernel: a label is ("label", name), an instruction (opcode, operands)."""
    name, body = None, []
    for line in asm.splitlines():
        line = line.split(";")[0].split("//")[0].rstrip()
        m = re.match(r"^([A-Za-z_.$][\w.$]*):$", line)
        if m and m[1].startswith("_Z"):
            name, body = m[1], []
        elif m and name:
            body.append(("label", m[1]))
        elif line.strip().startswith(".Lfunc_end") or re.match(r"^\s*\.end_amdhsa_kernel|^\s*\.size", line):
            if name and body:
                yield name, body
            name = None
        elif name and re.match(r"^\s+[a-z]\w*", line) and not line.strip().startswith("."):
            op, _, rest = line.strip().partition(" ")
            body.append((op, rest.strip()))


def barriers_with_pending_writes(body):
    """Places of the barriers that some path reaches with an LDS write that no wait has covered.

    The state before an instruction is the least number of LDS operations that any path has issued since its last
    uncovered write (None: every write is covered).  They complete in order, so that a wait for at most n outstanding
    ones covers the write if n is no larger."""
    at = {a: i for i, (op, a) in enumerate(body) if op == "label"}
    state, todo, bad = {0: None}, [0], set()

    def flow(i, s):
        if i >= len(body):
            return
        old = state.get(i, "new")
        new = s if old == "new" or old is None else old if s is None else min(old, s)
        if old == "new" or new != old:
            state[i] = new
            todo.append(i)

    while todo:
        i = todo.pop()
        s, (op, arg) = state[i], body[i]
        if op == "s_swappc_b64":
            raise AssertionError("a call, which this does not follow")
        if op.startswith("ds_") and not READS.match(op):
            s = 0
        elif op.startswith("ds_") and s is not None:
            s = min(s + 1, 15)
        elif op == "s_waitcnt":
            m = re.search(r"lgkmcnt\((\d+)\)", arg)
            if m and s is not None and int(m[1]) <= s:
                s = None
        elif op == "s_barrier" and s is not None:
            bad.add(i)
        if op == "s_endpgm":
            continue
        if op == "s_branch":
            flow(at[arg], s)
            continue
        if op == "s_setpc_b64":      # a far branch: its target is in the additions before it
            flow(at[re.search(r"\((\.LBB\w+)-", body[i - 1][1])[1]], s)
            continue
        if op.startswith("s_cbranch"):
            flow(at[arg], s)
        flow(i + 1, s)
    return sorted(bad)


def test_the_search_itself():
    write, read, bar, end = ("ds_write_b128", "v1, v[2:5]"), ("ds_read_b128", "v[2:5], v1"), ("s_barrier", ""), ("s_endpgm", "")
    wait = lambda n: ("s_waitcnt", f"lgkmcnt({n})")  # noqa: E731
    assert barriers_with_pending_writes([write, bar, end]) == [1]
    assert barriers_with_pending_writes([write, wait(0), bar, end]) == []
    assert barriers_with_pending_writes([write, ("s_waitcnt", "vmcnt(0)"), bar, end]) == [2]
    assert barriers_with_pending_writes([write, read, read, wait(2), bar, end]) == []
    assert barriers_with_pending_writes([write, read, read, wait(3), bar, end]) == [4]
    around = [write, ("s_cbranch_scc1", "over"), read, wait(0), ("label", "over"), bar, end]
    assert barriers_with_pending_writes(around) == [5]
    loop = [("label", "top"), bar, write, ("s_cbranch_scc0", "top"), wait(0), bar, end]
    assert barriers_with_pending_writes(loop) == [1]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "mx.s")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "asm", "mx_barriers.hip")
    cmd = [build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", src, "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-4000:]
    return open(out).read()


def test_no_barrier_with_writes_on_their_way(asm):
    found, kernels = {}, 0
    for name, body in functions(asm):
        if not re.search(r"few_kernel|few_redo_kernel|chunk_attn_kernel|chunk_redo_kernel", name):
            continue
        assert any(op == "s_barrier" for op, _ in body), name
        kernels += 1
        bad = barriers_with_pending_writes(body)
        if bad:
            found[name] = len(bad)
    assert kernels == 7, kernels
    assert not found, found
