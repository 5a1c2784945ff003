"""Properties of the generated code of the kernels over pages that their sources rely on and cannot express (CPU only): registers of LDS
reads that are waited for by hand are not touched before the wait, and nothing is kept in scratch (a reload would wait for
every tile in flight)."""
import re
import shutil

import pytest

from test_kernel_asm import device_code, registers

needs_hipcc = pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not found")


def touched_too_early(body):
    """(vector LDS reads of asm statements, instructions that name a read's registers before a wait covers it), along every path
    through the code.  LDS reads return in order; a wait for n leaves the n newest operations."""
    blocks, cur, in_asm, reads = [], ["entry", []], False, 0
    for line in body.splitlines():
        if "#ASMSTART" in line or "#ASMEND" in line:
            in_asm = "#ASMSTART" in line
            continue
        code = line.split(";")[0].strip()
        label = re.match(r"(\.L\w+):", code)
        if label:
            blocks.append(cur)
            cur = [label.group(1), []]
        elif code and not code.startswith("."):
            cur[1].append((code, in_asm))
            reads += in_asm and code.startswith("ds_read")
            if code.startswith(("s_cbranch", "s_branch", "s_endpgm")):
                blocks.append(cur)
                cur = [None, []]
    blocks.append(cur)
    at = {b[0]: i for i, b in enumerate(blocks) if b[0]}
    seen, todo, bad = [set() for _ in blocks], [(0, ())], set()
    while todo:
        i, pending = todo.pop()
        if i >= len(blocks) or pending in seen[i]:
            continue
        seen[i].add(pending)
        pending, after = list(pending), [i + 1]                # LDS and scalar operations in issue order: a read's registers or None
        for code, in_asm in blocks[i][1]:
            op, _, args = code.partition(" ")
            count = re.search(r"lgkmcnt\((\d+)\)", args) if op == "s_waitcnt" else None
            if count:
                pending = pending[len(pending) - min(len(pending), int(count.group(1))):]
            if op == "s_waitcnt":
                continue
            names = registers(args, "va")
            if any(p and p & names for p in pending):
                bad.add(code)
            if op.startswith("ds_read") and in_asm:
                pending.append(frozenset(registers(args.split(",")[0], "va")))
            elif op.startswith(("ds_", "s_load", "s_buffer_load")):
                pending.append(None)
            if op.startswith(("s_cbranch", "s_branch")):
                after = [at[args.strip()]] + ([i + 1] if op.startswith("s_cbranch") else [])
            elif op == "s_endpgm":
                after = []
        while pending and pending[0] is None:
            pending.pop(0)
        todo += [(x, tuple(pending)) for x in after]
    return reads, sorted(bad)


@needs_hipcc
def test_rows_kernels():
    kernels, scratch = device_code("paged_rows.hip")
    mine = {k: v for k, v in kernels.items() if "paged_rows_kernel" in k}
    assert len(mine) == 11, sorted(kernels)
    for k, body in mine.items():
        found, bad = touched_too_early(body)
        assert found >= 8 and not bad, (k, found, bad[:5])
        assert scratch[k] == 0, scratch


@needs_hipcc
@pytest.mark.parametrize("name", ["paged_fwd", "paged_mixed"])
def test_fwd_kernels(name):
    kernels, scratch = device_code(name + ".hip")
    mine = {k: v for k, v in kernels.items() if name + "_kernel" in k}
    assert len(mine) == 4, sorted(kernels)
    for k, body in mine.items():
        assert scratch[k] == 0, scratch
        found, bad = touched_too_early(body)
        assert found >= 64 and not bad, (k, found, bad[:5])
        # a V fragment's two reads fill one register quadruple, which the product reads as it stands
        reads = [int(x) for x in re.findall(r"ds_read_b64_tr_b16 v\[(\d+):\d+\]", body)]
        assert len(reads) % 2 == 0 and all(b == a + 2 for a, b in zip(reads[0::2], reads[1::2]))
        operands = {int(x) for x in re.findall(r"v_mfma_f32_(?:32x32x16|16x16x32)_bf16 [av]\[\d+:\d+\], v\[(\d+):\d+\], v\[", body)}
        assert set(reads[0::2]) <= operands, sorted(set(reads[0::2]) - operands)


def test_the_check_follows_branches():
    read = "\t;;#ASMSTART\n\tds_read_b128 v[4:7], v1 offset:0\n\t;;#ASMEND\n"
    use, wait = "\tv_mov_b32_e32 v0, v5\n", "\ts_waitcnt lgkmcnt(0)\n"
    jump = "\ts_cbranch_scc1 .LBB0_1\n"
    assert touched_too_early(read + jump + wait + use + ".LBB0_1:\n" + wait + use + "\ts_endpgm\n") == (1, [])
    assert touched_too_early(read + jump + wait + use + "\ts_endpgm\n.LBB0_1:\n" + use + "\ts_endpgm\n") == (1, [use.strip()])
    assert touched_too_early(read + "\ts_branch .LBB0_2\n.LBB0_1:\n" + use + "\ts_endpgm\n.LBB0_2:\n" + wait + use + "\ts_endpgm\n") == (1, [])
