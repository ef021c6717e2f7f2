"""The compiled kernels of quantized language models: LDS that is read before a workgroup barrier is overwritten behind it, so
that no read may be on its way where a wave arrives.  Found in the library's own code objects, without a GPU."""
import os
import re
import shutil
import subprocess

import pytest

import paper_1806_08342_amd as qnn

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def instructions(path, kernel):
    """{symbol: [(address, text, target of a branch or None)]} of the kernels whose names contain `kernel`."""
    text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout
    found, into = {}, None
    for line in text.splitlines():
        head = re.match(r"^[0-9a-f]+ <(\S+)>:", line)
        if head:
            into = found.setdefault(head.group(1), []) if kernel in head.group(1) else None
            continue
        m = re.match(r"^\t(\S.*?)\s*// ([0-9A-F]+):(.*)", line)
        if m and into is not None:
            target = re.search(r"<\S+?\+0x([0-9a-f]+)>", m.group(1) + m.group(3))
            into.append((int(m.group(2), 16), m.group(1), int(target.group(1), 16) if target else None))
    return found


def merged(a, b):
    """Both lists of requests on their way, youngest last: a read where either has one."""
    if a is None:
        return b
    n = max(len(a), len(b))
    a, b = (" ",) * (n - len(a)) + a, (" ",) * (n - len(b)) + b
    return tuple("read" if "read" in pair else max(pair) for pair in zip(a, b))


def reads_at_barriers(code):
    """{offset of a barrier: LDS reads that may be on their way at it}, over all paths."""
    base, index = code[0][0], {at: i for i, (at, _, _) in enumerate(code)}
    states, todo, at_barrier = [None] * len(code), [(0, ())], {}
    while todo:
        i, now = todo.pop()
        while i < len(code):
            now = merged(states[i], now)
            if now == states[i]:
                break
            states[i] = now
            at, text, target = code[i]
            name = text.split()[0]
            if name.startswith(("ds_", "s_load", "s_buffer_load")):
                now = (now + ("read" if "read" in name else "other",))[-64:]
            elif name == "s_waitcnt" and "lgkmcnt" in text:
                left = int(re.search(r"lgkmcnt\((\d+)\)", text).group(1))
                now = now[max(0, len(now) - left):]
            elif name == "s_barrier":
                at_barrier[at - base] = now.count("read")
            elif name == "s_endpgm":
                break
            elif name == "s_branch":
                i = index[base + target]
                continue
            elif name.startswith("s_cbranch"):
                todo.append((index[base + target], now))
            i += 1
    return at_barrier


@pytest.fixture(scope="module")
def objects(tmp_path_factory):
    qnn.load_library()
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    where = tmp_path_factory.mktemp("objects")
    shutil.copy(qnn.library_path(), where / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=where, check=True, capture_output=True)
    paths = sorted(p for p in where.iterdir() if "gfx950" in p.name)
    assert paths
    return [(p, p.read_bytes()) for p in paths]


@pytest.mark.parametrize("kernel", ["w4_tile_kernel", "w4_parts_kernel", "attend_prompt_kernel", "attend_wide_kernel"])
def test_no_read_is_on_its_way_at_a_barrier(objects, kernel):
    seen = 0
    for path, contents in objects:
        if kernel.encode() not in contents:
            continue
        for symbol, code in instructions(str(path), kernel).items():
            if not code or symbol.endswith(".kd"):
                continue
            at_barrier = reads_at_barriers(code)
            assert at_barrier and not any(at_barrier.values()), (symbol, at_barrier)
            seen += 1
    assert seen >= 4
