"""The compiled kernels of 8-bit floating point: what a matrix instruction writes is not read before it is there (the compiler's waits for it do not
always reach over a branch), and no read of LDS is on its way at a barrier behind which its place is filled again.  Found in the library's own
code objects, without a GPU."""
import re

import pytest

from test_lm_device_code import instructions, objects, reads_at_barriers  # noqa: F401 (a fixture among them)

PASSES = {"16x16x128_f8f6f4": 8, "32x32x64_f8f6f4": 16, "16x16x32_bf16": 4, "32x32x16_bf16": 8}  # four cycles each


def registers(operand):
    m = re.match(r"^-?\|?v\[(\d+):(\d+)\]", operand) or re.match(r"^-?\|?v(\d+)\b", operand)
    return frozenset(range(int(m.group(1)), int(m.group(m.lastindex)) + 1)) if m else frozenset()


def parsed(text):
    """(name, registers read, registers written, operands)"""
    name, _, rest = text.partition(" ")
    operands = [o.strip() for o in rest.split(",")] if rest else []
    each = [registers(o) for o in operands]
    every = frozenset().union(*each)
    if name.startswith(("ds_write", "global_store", "buffer_store", "flat_store", "scratch_store", "v_permlane", "v_swap")):
        return name, every, frozenset(), operands
    reads = frozenset().union(*each[1:])
    if name.startswith("v_mfma"):
        reads = each[1] | each[2]  # (what is added to follows in order)
    elif name.startswith("v_fmac"):
        reads = every
    return name, reads, each[0] if each else frozenset(), operands


def read_too_early(code):
    """Instructions that may read what a matrix instruction has not written yet, over all paths."""
    base, index = code[0][0], {at: i for i, (at, _, _) in enumerate(code)}
    lines, found = [parsed(text) for _, text, _ in code], []
    for i, (name, _, written, _) in enumerate(lines):
        if not name.startswith("v_mfma"):
            continue
        passes = next(v for k, v in PASSES.items() if k in name)
        needed = passes + 4  # wait states between it and a vector instruction that reads its result
        seen, todo = {}, [(i + 1, 0, written)]
        while todo:
            j, waited, live = todo.pop()
            while j < len(code) and waited < needed and live and seen.get((j, live), needed) > waited:
                seen[j, live] = waited
                other, reads, writes, operands = lines[j]
                if reads & live:
                    found.append((name, code[j][1], waited, needed))
                    break
                live = live - writes
                if other.startswith("v_mfma"):
                    waited = max(waited, passes)  # there is one matrix unit: it begins when the first has ended
                if other == "s_endpgm":
                    break
                if other.startswith(("s_branch", "s_cbranch")):
                    to = index[base + code[j][2]]
                    if other == "s_branch":
                        j, waited = to, waited + 1
                        continue
                    todo.append((to, waited + 1, live))
                waited += int(operands[0], 0) + 1 if other == "s_nop" else 1
                j += 1
    return found


def kernels(objects, name):  # noqa: F811
    for path, contents in objects:
        if name.encode() in contents:
            for symbol, code in instructions(str(path), name).items():
                if code and not symbol.endswith(".kd"):
                    yield symbol, code


@pytest.mark.parametrize("kernel, least", [("f8_tile_kernel", 3), ("f8_rows_kernel", 18), ("moe_up_kernel", 5), ("moe_down_kernel", 2), ("moe_down_wide_kernel", 1)])
def test_products_are_read_when_they_are_there(objects, kernel, least):  # noqa: F811
    seen = 0
    for symbol, code in kernels(objects, kernel):
        assert any(text.startswith("v_mfma") for _, text, _ in code), symbol
        early = read_too_early(code)
        assert not early, (symbol, early[:3])
        seen += 1
    assert seen >= least


def test_an_early_read_is_found():
    mfma = "v_mfma_f32_16x16x32_bf16 v[0:3], v[4:7], v[8:11], 0"
    code = lambda *texts: [(4 * i, t, None) for i, t in enumerate(texts)]  # noqa: E731
    assert read_too_early(code(mfma, "s_nop 6", "v_fmac_f32_e32 v20, v3, v21", "s_endpgm"))
    assert not read_too_early(code(mfma, "s_nop 7", "v_fmac_f32_e32 v20, v3, v21", "s_endpgm"))
    assert read_too_early(code(mfma, "global_store_dword v[30:31], v2, off", "s_endpgm"))
    assert not read_too_early(code(mfma, "v_mov_b32_e32 v3, v9", "v_add_f32_e32 v20, v3, v21", "s_endpgm"))
    over = code(mfma, "s_cbranch_scc1 x", "s_nop 7", "v_add_f32_e32 v20, v0, v21", "s_endpgm")
    over[1] = (4, "s_cbranch_scc1 x", 12)
    assert read_too_early(over)


@pytest.mark.parametrize("kernel, least", [("f8_tile_kernel", 3), ("moe_down_wide_kernel", 1)])
def test_no_read_is_on_its_way_at_a_barrier_behind_which_its_place_is_filled(objects, kernel, least):  # noqa: F811
    seen = 0
    for symbol, code in kernels(objects, kernel):
        at_barrier = reads_at_barriers(code)
        assert at_barrier and not any(at_barrier.values()), (symbol, at_barrier)
        seen += 1
    assert seen >= least


@pytest.mark.parametrize("kernel, newest, of_a_pass, least", [("moe_down_kernel", 8, 6, 2), ("moe_down_wide_kernel", 5, 5, 1)])
def test_copies_are_counted_as_the_waits_for_them_assume(objects, kernel, newest, of_a_pass, least):  # noqa: F811
    # moe_down_kernel waits until all but the newest eight copies have arrived: six of a pass over its loop and two of the one before; the wide one,
    # before it requests more, until all but the last pass's five have
    seen = 0
    for symbol, code in kernels(objects, kernel):
        texts = [text for _, text, _ in code]
        waits = [i for i, t in enumerate(texts) if re.fullmatch(rf"s_waitcnt vmcnt\({newest}\)", t)]
        assert len(waits) == 1, symbol
        first_product = next(i for i, t in enumerate(texts) if t.startswith("v_mfma"))
        assert waits[0] < first_product
        base = code[0][0]
        # the loop: from what a later branch goes back to, before the wait, to the last such branch
        backs = [(base + to, i) for i, (_, t, to) in enumerate(code) if i > waits[0] and t.startswith(("s_cbranch", "s_branch")) and to is not None and base + to < code[waits[0]][0]]
        index = {at: i for i, (at, _, _) in enumerate(code)}
        begin, end = max((index[to], i) for to, i in backs)
        memory = [t for t in texts[begin:end] if t.startswith(("global_", "buffer_", "flat_", "scratch_"))]
        assert len(memory) == of_a_pass and all(t.startswith("buffer_load_dwordx4") and t.endswith(" lds") for t in memory), (symbol, memory)
        seen += 1
    assert seen >= least
