"""Reads of matrix instructions' results that come too early, found in compiled kernels' assembly.

The hardware does not hold an ordinary instruction back that reads what an MFMA has still to write: a number of others has to be issued in
between (passes + 4 on this GPU for the 16-bit and 8-bit types with more than two passes, passes + 2 for fp32).  The compiler puts s_nop
there, but where a branch that may be skipped lies between the two it has been seen to count the longer way only.  This follows every way
through a kernel and keeps, for each register, how many instructions are still missing."""
import re

# passes of the shapes in use, and what the result needs beyond them
NEED = [("32x32x16_f16", 12), ("32x32x16_bf16", 12), ("16x16x32_f16", 8), ("16x16x32_bf16", 8), ("32x32x2_f32", 18), ("16x16x4_f32", 10)]
REG = re.compile(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b")


def registers(text):
    out = []
    for m in REG.finditer(text):
        if m.group(1):
            out += [(m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1)]
        else:
            out.append((m.group(4), int(m.group(5))))
    return out


def kernels(lines):
    """(name, lines) of each kernel in a file of assembly."""
    name = body = None
    for l in lines:
        m = re.match(r"^(_ZN\S+kernel\S*):", l)
        if m:
            name, body = m.group(1), []
        elif name and ".amdhsa_kernel" in l:
            yield name, body
            name = None
        elif name:
            body.append(l)


def blocks_of(body):
    """Blocks of instructions, which end at labels and at branches (what follows a branch that may be skipped has no label of its own),
    and the names of those that follow each."""
    blocks, at = {"": []}, ""
    for l in body:
        m = re.match(r"^(\.LBB\S+):", l)
        s = "" if m else l.split(";")[0].strip()
        if m:
            at = m.group(1)
            blocks[at] = []
        elif s and not s.startswith("."):
            blocks[at].append(s)
            if s.startswith(("s_cbranch", "s_branch", "s_endpgm")):
                at = f"behind {len(blocks)}"
                blocks[at] = []
    names, follow = list(blocks), {}
    for i, b in enumerate(names):
        last = blocks[b][-1] if blocks[b] else ""
        follow[b] = [last.split()[-1]] if last.startswith(("s_cbranch", "s_branch")) else []
        if not last.startswith(("s_branch", "s_endpgm")) and i + 1 < len(names):
            follow[b].append(names[i + 1])
    return blocks, follow


def walk(instructions, missing, early=None, busy=False):
    """What is missing behind these instructions; early: gets those that read or overwrite a result too soon.  busy: a matrix instruction
    keeps its unit for its passes, so that the next one issues as many states later (the compiler counts one)."""
    missing, free = dict(missing), 0
    for s in instructions:
        op, rest = s.split()[0], s[len(s.split()[0]):]
        matrix = op.startswith(("v_mfma", "v_smfmac"))
        if matrix and busy:
            missing, free = {r: k - free for r, k in missing.items() if k > free}, 0
        if early is not None and op.startswith(("v_", "ds_", "global_", "buffer_", "scratch_", "flat_")):
            # (a sum that goes on in the next product is the hardware's to order)
            text = ",".join(rest.split(",")[1:3]) if matrix else rest
            early += [(s, r, missing[r]) for r in set(registers(text)) if missing.get(r, 0) > 0]
        step = int(rest.strip(), 0) + 1 if op == "s_nop" else 1
        missing, free = {r: k - step for r, k in missing.items() if k > step}, max(free - step, 0)
        if matrix:
            need = [n for shape, n in NEED if shape in op]
            assert need, f"unknown shape: {op}"
            missing.update((r, need[0]) for r in registers(rest.split(",")[0]))
            free = need[0] - (2 if op.endswith("_f32") else 4) - 1
    return missing


def early_reads(body, busy=False):
    blocks, follow = blocks_of(body)
    state, todo, reached = {b: {} for b in blocks}, [""], {""}
    while todo:
        b = todo.pop()
        out = walk(blocks[b], state[b], busy=busy)
        for to in follow[b]:
            worse = {r: k for r, k in out.items() if state[to].get(r, 0) < k}
            if worse or to not in reached:
                state[to].update(worse)
                reached.add(to)
                todo.append(to)
    early = []
    for b in blocks:
        walk(blocks[b], state[b], early, busy)
    return early
