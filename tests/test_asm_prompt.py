"""Static check of the attention over packed sequences' explicitly waited LDS reads (CPU only).

The bf16 kernels issue LDS reads as inline assembly and wait for them with `s_waitcnt lgkmcnt(n)`;
the compiler takes a read's registers as written the moment it is issued.  This test walks the gfx950
assembly of every instantiation along all its branches with the queue of LDS operations under way
(they complete in order) and checks that no instruction reads or writes the registers of a read that
may still be coming.  Tiles come by loads whose LDS address is in m0: nothing else may use m0, and no
instantiation of a kernel with two waves a SIMD may spill (a reload would wait for the next tile).
"""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCES = ["prompt_attn.hip"]


def _regs(text):
    out = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {(kind, i) for i in range(int(a), int(b) + 1)}
    for kind, a in re.findall(r"(?<![\w\[:.])([va])(\d+)\b", text):
        out.add((kind, int(a)))
    return out


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not os.path.exists(HIPCC) and not shutil.which("hipcc"):
        pytest.skip("hipcc not available")
    found = {}
    for src in SOURCES:
        out = tmp_path_factory.mktemp("asm") / (src + ".s")
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
                        "-packed-fp32-ops", f"-I{os.path.join(ROOT, 'include')}", "--cuda-device-only", "-S",
                        os.path.join(ROOT, "paper_2609_31224_amd", "csrc", src), "-o", str(out)], check=True, capture_output=True)
        name, body = None, []
        for line in open(out):
            if re.match(r"^_ZN\w+:", line):
                name, body = line.split(":")[0], []
            elif name and line.startswith("; ScratchSize:"):
                found[name] = (body, int(line.split()[-1]))
                name = None
            elif name:
                body.append(line.split(";")[0].strip())
    assert len(found) >= 3 * 2 * 2 * 2 * 4
    return found


def _blocks(body):
    """Basic blocks: label or start -> (instructions, successors)."""
    starts, blocks, cur = {}, [[]], None
    for l in body:
        m = re.match(r"^(\.LBB\w+):$", l)
        if m:
            if blocks[-1]:
                blocks.append([])
            starts[m.group(1)] = len(blocks) - 1
            continue
        if not l or l.startswith((".", "_Z")):
            continue
        blocks[-1].append(l)
        if l.startswith(("s_branch", "s_cbranch", "s_endpgm")):
            blocks.append([])
    out = []
    for i, b in enumerate(blocks):
        succ = [i + 1] if i + 1 < len(blocks) else []
        if b:
            m = re.match(r"s_c?branch\S* (\.LBB\w+)", b[-1])
            if m:
                succ = [starts[m.group(1)]] + ([i + 1] if b[-1].startswith("s_cbranch") else [])
            if b[-1].startswith("s_endpgm"):
                succ = []
        out.append((b, succ))
    return out


def _step(line, queue):
    """The queue after `line`, or None where the line touches registers that are still coming."""
    m = re.search(r"s_waitcnt.*lgkmcnt\((\d+)\)", line)
    if m:
        n = int(m.group(1))
        return queue[len(queue) - n:] if n < len(queue) else queue
    if line.startswith("s_waitcnt"):
        return queue
    coming = frozenset().union(*queue) if queue else frozenset()
    if coming & _regs(line):
        return None
    if line.startswith("ds_"):
        dest = line.split(",")[0] if re.match(r"ds_(read|swizzle|bpermute|permute)", line) else ""
        return (queue + (frozenset(_regs(dest)),))[-16:]
    return queue


def test_lds_reads_are_waited_for(kernels):
    for name, (body, _) in kernels.items():
        blocks = _blocks(body)
        seen, todo, reads = set(), [(0, ())], 0
        while todo:
            i, queue = todo.pop()
            if (i, queue) in seen:
                continue
            seen.add((i, queue))
            assert len(seen) < 20000, name
            for l in blocks[i][0]:
                reads += l.startswith("ds_read")
                after = _step(l, queue)
                assert after is not None, (name, l)
                queue = after
            todo += [(s, queue) for s in blocks[i][1]]
        assert reads or "prompt_join" in name or "prompt_add" in name, name


def test_a_missing_wait_is_found():
    """The check itself: a use before its wait, and one after too weak a wait."""
    def walk(lines):
        q = ()
        for l in lines:
            q = _step(l, q)
            if q is None:
                return l
        return None
    two = ["ds_read_b128 v[0:3], v9", "ds_read_b128 v[4:7], v9"]
    assert walk(two + ["s_waitcnt lgkmcnt(1)", "v_add_f32_e32 v10, v0, v1", "s_waitcnt lgkmcnt(0)", "v_add_f32_e32 v10, v4, v5"]) is None
    assert walk(two + ["s_waitcnt lgkmcnt(1)", "v_add_f32_e32 v10, v4, v5"]) == "v_add_f32_e32 v10, v4, v5"
    assert walk(two + ["v_mov_b32_e32 v20, v2"]) is not None
    assert walk(two + ["v_mfma_f32_32x32x16_bf16 a[0:15], v[6:9], v[20:23], a[0:15]"]) is not None


def test_m0_and_scratch(kernels):
    for name, (body, scratch) in kernels.items():
        for a, b in zip(body, body[1:] + [""]):
            if re.search(r"\bm0\b", a):
                assert a.startswith("s_mov_b32 m0,") and b.startswith("s_nop"), (name, a, b)
        narrow = "IfLi128E" in name      # fp32 rows of 512 bytes: one wave a SIMD, 512 registers
        assert scratch == 0, (name, scratch, narrow)
