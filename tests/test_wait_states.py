"""Wait states between a matrix instruction and the first other use of its result, along
every path through the built library's kernels.

The result of a matrix instruction of P passes may be read or overwritten by a vector
instruction, stored, or read as another product's A or B operand P + 3 wait states later
(P + 2 for fp32 operands); the hardware does not wait by itself, and the compiler fills in
what is missing.  hipcc was found to leave too few where a taken branch lies between.
A wait state is the time of one instruction (a pass); a matrix instruction waits
until the one before it has gone through its passes, since they share one unit.
"""
import collections
import os
import re
import subprocess

import pytest

from paper_2606_07317_amd import build

PASSES = {"32x32x16_bf16": 8, "16x16x32_bf16": 4, "32x32x2_f32": 16, "16x16x4_f32": 8}

Op = collections.namedtuple("Op", "name args words at")


def _need(name):
    """(passes, wait states) of a matrix instruction; None for other instructions."""
    if not name.startswith("v_mfma"):
        return None
    for shape, passes in PASSES.items():
        if name in ("v_mfma_f32_" + shape, "v_mfma_f32_" + shape.replace("_f32", "f32")):
            return passes, passes + (2 if shape.endswith("_f32") else 3)
    raise AssertionError("passes of %s are not known here" % name)


def _registers(text):
    found = set()
    for kind, a, b in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        found |= {(kind, i) for i in range(int(a), int(b) + 1)}
    return found | {(kind, int(i)) for kind, i in re.findall(r"\b([va])(\d+)\b", text)}


def _operands(op):
    """(registers read, registers written) of an instruction other than a matrix product."""
    first, _, rest = op.args.partition(",")
    if op.name.startswith("v_cmp") or op.name.startswith("v_readfirstlane"):
        return _registers(op.args), set()
    if op.name.startswith("v_"):
        both = op.name.startswith(("v_fmac", "v_mac", "v_swap"))
        return _registers(op.args if both else rest), _registers(first)
    if "load" in op.name and "lds" not in op.args.split():
        return _registers(rest), _registers(first)
    if op.name.startswith("ds_read"):
        return _registers(rest), _registers(first)
    return _registers(op.args), set()


def kernels(listing):
    """{name: [Op]} of a disassembly."""
    found, body = {}, None
    for line in listing.splitlines():
        head = re.match(r"^[0-9a-f]+ <(.*)>:", line)
        if head:
            body = found.setdefault(head.group(1), [])
            continue
        m = re.match(r"^\s+(\S+)\s*(.*?)\s*//\s*([0-9A-F]+):((?: [0-9A-F]{8})+)", line)
        if m and body is not None:
            body.append(Op(m.group(1), m.group(2), len(m.group(4).split()), int(m.group(3), 16)))
    return found


def short_paths(ops):
    """(matrix instruction, use, wait states, wait states due) of every use that comes too soon."""
    index = {op.at: i for i, op in enumerate(ops)}
    found = set()
    for i, op in enumerate(ops):
        due = _need(op.name)
        if due is None:
            continue
        passes, need = due
        result = frozenset(_registers(op.args.split(",")[0]))
        todo, seen = [(i + 1, 0, passes - 1, result)], set()
        while todo:
            j, states, busy, regs = todo.pop()
            # `states` have gone by; the unit is free from state `busy` on
            while j < len(ops) and states < need and regs and (j, states, busy, regs) not in seen:
                seen.add((j, states, busy, regs))
                o = ops[j]
                again = _need(o.name)
                if again is not None:
                    parts = [_registers(x) for x in re.findall(r"[va]\[[^\]]*\]|[^,\s]+", o.args)]
                    if (parts[1] | parts[2]) & regs:
                        if max(states, busy) < need:
                            found.add((i, j, states, need))
                        break
                    states = max(states, busy) + 1
                    busy = states - 1 + again[0]
                    regs -= parts[0]
                    j += 1
                    continue
                if o.name == "s_nop":
                    states += int(o.args.split()[0], 0) + 1
                elif o.name == "s_endpgm":
                    break
                elif o.name.startswith(("s_cbranch", "s_branch")):
                    states += 1
                    off = int(o.args.split()[0])
                    target = o.at + 4 * o.words + 4 * (off - 65536 if off > 32767 else off)
                    todo.append((index[target], states, busy, regs))
                    if o.name == "s_branch":
                        break
                else:
                    if o.name.startswith(("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")):
                        read, written = _operands(o)
                        if (read | written) & regs:
                            found.add((i, j, states, need))
                            break
                    states += 1
                j += 1
    return [(ops[i], ops[j], states, need) for i, j, states, need in sorted(found)]


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    tool = os.path.join(rocm, "llvm", "bin", "llvm-objdump")
    if not os.path.exists(tool):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(build.LIB):
        build.build()
    where = tmp_path_factory.mktemp("code")
    os.symlink(build.LIB, where / "lib.so")
    subprocess.run([tool, "--offloading", "lib.so"], cwd=where, check=True, capture_output=True)
    found = {}
    for name in sorted(os.listdir(where)):
        if name.endswith("gfx950"):
            text = subprocess.run([tool, "-d", name], cwd=where, check=True, capture_output=True, text=True)
            found.update(kernels(text.stdout))
    return found


def test_no_result_is_used_too_soon(library):
    with_products = {n: ops for n, ops in library.items() if any(o.name.startswith("v_mfma") for o in ops)}
    for part in ("walk_kernel", "keys_kernel", "record_kernel", "proj_kernel"):
        assert any(part in n for n in with_products), part
    short = {n: short_paths(ops) for n, ops in with_products.items()}
    short = {n: s for n, s in short.items() if s}
    assert not short, "\n".join("%s: %s" % (n, s[0]) for n, s in short.items())


PRODUCT = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]"


def _listing(*lines):
    """A listing of one kernel; every instruction is taken as one word."""
    return "0000 <k>:\n" + "\n".join(" %s // %012X: 00000000" % (x, 4 * i) for i, x in enumerate(lines))


@pytest.mark.parametrize("between,short", [
    (["s_nop 6"], False),
    (["s_nop 5"], True),
    (["v_mov_b32_e32 v20, v21"] * 7, False),
    (["v_mov_b32_e32 v20, v21"] * 6, True),
    # the branch jumps over the waiting
    (["s_cbranch_scc1 1", "s_nop 6"], True),
    (["s_cbranch_scc1 1", "s_nop 6", "s_nop 5"], False),
    # a second product has to wait for the unit
    (["v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], v[4:7]", "s_nop 2"], False),
    (["v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], v[4:7]", "s_nop 1"], True),
    # the result goes on as an operand
    (["s_nop 2", "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], v[4:7]", "s_nop 15"], True),
    (["s_nop 6", "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], v[4:7]", "s_nop 15"], False),
])
def test_the_scan_finds_planted_places(between, short):
    ops = kernels(_listing(PRODUCT, *between, "v_add_f32_e32 v30, v2, v31", "s_endpgm"))["k"]
    assert bool(short_paths(ops)) == short


@pytest.mark.parametrize("use", ["ds_write_b32 v30, v1", "buffer_store_dwordx4 v[0:3], v30, s[0:3], 0 offen",
                                 "v_mov_b32_e32 v3, v31", "v_cmp_gt_f32_e32 vcc, v3, v31"])
def test_the_scan_sees_every_kind_of_use(use):
    assert short_paths(kernels(_listing(PRODUCT, use, "s_endpgm"))["k"])
    assert not short_paths(kernels(_listing(PRODUCT, "s_nop 6", use, "s_endpgm"))["k"])
