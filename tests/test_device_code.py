"""What the compiler made of the kernels: two mistakes of its that gave wrong values here, looked for in the built library's
own code on the CPU.

Matrix results.  A result of a matrix instruction must not be read or written over for some cycles.  The compiler
inserts waits, but looks back over one side of a branch only and misses the shorter one.  Here every path is walked.

Spills.  Where two sides of a branch join, lanes are switched on again by an instruction at the head of the block.  A
register that is stored to scratch memory before it is saved for some of the lanes only."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2307_12983_amd.binding import LIB_PATH

OBJDUMP = next((p for p in (os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib", "llvm", "bin", "llvm-objdump"),
                            shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
# cycles between a matrix instruction and a use of its result by any other
WAIT = {"f32_16x16x4_f32": 10, "f32_32x32x2_f32": 18, "f32_16x16x32_bf16": 7, "f32_16x16x32_f16": 7, "f32_32x32x16_f16": 11}


def code_objects():
    """The gfx950 code objects in the library's offload bundles."""
    data = open(LIB_PATH, "rb").read()
    at = data.find(b"__CLANG_OFFLOAD_BUNDLE__")
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count if count < 8 else 0):          # the linker's copy of the mark has no entries
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            triple = data[entry + 24:entry + 24 + length]
            entry += 24 + length
            if triple.endswith(b"gfx950") and size:
                yield data[at + offset:at + offset + size]
        at = data.find(b"__CLANG_OFFLOAD_BUNDLE__", at + 24)


def parse(text):
    """{function: [(address, mnemonic, operands)]} of a disassembly."""
    functions, current = {}, None
    for line in text.splitlines():
        m = re.match(r"^[0-9a-f]+ <(\S+)>:$", line)
        if m:
            current = functions.setdefault(m.group(1), [])
            continue
        m = re.match(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+): ", line)
        if m and current is not None:
            current.append((int(m.group(3), 16), m.group(1), m.group(2)))
    return functions


def blocks_of(code):
    """Basic blocks as ranges of `code`, and where each goes on."""
    place = {a: i for i, (a, _, _) in enumerate(code)}
    jumps = {}
    for i, (address, op, args) in enumerate(code):
        if op.startswith(("s_branch", "s_cbranch")):
            offset = int(args.split()[0])
            jumps[i] = place[address + 4 + 4 * (offset - 65536 if offset > 32767 else offset)]
    starts = sorted({0, *jumps.values(), *(i + 1 for i in jumps)} - {len(code)})
    number = {s: n for n, s in enumerate(starts)}
    blocks = []
    for n, s in enumerate(starts):
        end = starts[n + 1] if n + 1 < len(starts) else len(code)
        last, to = code[end - 1][1], []
        if end - 1 in jumps:
            to.append(number[jumps[end - 1]])
        if not last.startswith(("s_branch", "s_endpgm", "s_setpc")) and end < len(code):
            to.append(n + 1)
        blocks.append((s, end, to))
    return blocks


def registers(operands):
    out = []
    for m in re.finditer(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)", operands):
        low, high = (int(m.group(2)), int(m.group(3))) if m.group(2) else (int(m.group(4)),) * 2
        out += [(m.group(1), i) for i in range(low, high + 1)]
    return out


def early_uses(code):
    """Instructions that read or write over a matrix result too early on some path."""
    steps = []
    for _, op, args in code:
        parts = args.split(", ")
        mfma = op.startswith("v_mfma")
        reads = writes = ()
        if mfma:                                            # an accumulator of the same kind is forwarded
            reads = registers(", ".join(parts[1:3]))
        elif op.startswith(("buffer_store", "global_store", "flat_store", "scratch_store", "ds_write")):
            reads = registers(args)
        elif op.startswith(("v_", "buffer_", "global_", "flat_", "scratch_", "ds_")):
            reads = registers(", ".join(parts[1:]))
            writes = registers(parts[0]) if op.startswith("v_") else ()
        results = [(r, WAIT.get(op[len("v_mfma_"):], 19)) for r in registers(parts[0])] if mfma else ()
        steps.append((int(args) + 1 if op == "s_nop" else 1, reads, writes, results))
    blocks, found = blocks_of(code), set()
    state, work = {0: {}}, [0]
    while work:
        n = work.pop()
        start, end, to = blocks[n]
        now = dict(state[n])
        for i in range(start, end):
            cycles, reads, writes, results = steps[i]
            if now:
                if any(r in now for r in reads) or any(r in now for r in writes):
                    found.add(i)
                now = {r: w - cycles for r, w in now.items() if w > cycles}
            now.update(results)
        for s in to:
            old = state.get(s)
            new = dict(old or {})
            for r, w in now.items():
                new[r] = max(w, new.get(r, 0))
            if new != old:
                state[s] = new
                work.append(s)
    return ["%s %s" % code[i][1:] for i in sorted(found)]


def masked_spills(code):
    """Stores to scratch memory at the head of a block, before that block switches lanes on again."""
    found = []
    for start, end, _ in blocks_of(code):
        pending = []
        for _, op, args in code[start:end]:
            if "saveexec" in op:
                pending = []
            elif op.startswith("scratch_store"):
                pending.append("%s %s" % (op, args))
            elif op == "s_or_b64" and args.startswith("exec, exec"):
                found += pending
                pending = []
    return found


@pytest.fixture(scope="module")
def functions():
    if OBJDUMP is None:
        pytest.skip("no llvm-objdump")
    out = {}
    for n, co in enumerate(code_objects()):
        text = subprocess.run([OBJDUMP, "-d", "/dev/stdin"], input=co, capture_output=True, check=True).stdout.decode()
        out.update({(n, name): code for name, code in parse(text).items() if code})
    return out


def test_no_matrix_result_is_used_too_early(functions):
    with_products = {k: c for k, c in functions.items() if any(op.startswith("v_mfma") for _, op, _ in c)}
    assert len(with_products) > 100
    bad = {k: early_uses(c) for k, c in with_products.items()}
    assert not {k: v[:3] for k, v in bad.items() if v}


def test_no_register_is_spilled_for_some_lanes_only(functions):
    assert not {k: v for k, v in ((k, masked_spills(c)) for k, c in functions.items()) if v}


def test_the_two_checks_see_what_they_look_for():
    def code(text):
        return parse("0 <f>:\n" + "\n".join("\t%s // %012X: 0" % (t, 4 * i) for i, t in enumerate(text)))["f"]
    # the branch leaves out the long wait
    early = code(["v_mfma_f32_16x16x4_f32 a[0:3], v0, v1, a[0:3]", "s_cbranch_scc1 1", "s_nop 15", "v_accvgpr_read_b32 v2, a3", "s_endpgm "])
    assert early_uses(early) == ["v_accvgpr_read_b32 v2, a3"]
    late = code(["v_mfma_f32_16x16x4_f32 a[0:3], v0, v1, a[0:3]", "s_cbranch_scc1 1", "s_nop 15", "s_nop 8", "v_accvgpr_read_b32 v2, a3", "s_endpgm "])
    assert early_uses(late) == []
    masked = code(["s_and_saveexec_b64 s[0:1], vcc", "s_cbranch_execz 1", "v_mov_b32_e32 v0, v1", "scratch_store_dword off, v2, off offset:20",
                   "s_or_b64 exec, exec, s[0:1]", "scratch_store_dword off, v3, off", "s_endpgm "])
    assert masked_spills(masked) == ["scratch_store_dword off, v2, off offset:20"]
