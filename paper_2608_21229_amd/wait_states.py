"""Checks an assembly listing for the wait states that matrix products written
as statements of assembly need, which the compiler's hazard recogniser does not
see:

* two wait states between a vector instruction, or a block's start, and a
  product that reads its result (an LDS read is waited for by the compiler);
* ``SETTLED`` of them between a product and any other instruction that touches
  its accumulators, along every path: each register's youngest age is carried
  over the branches until nothing changes.

An instruction is one wait state, ``s_nop n`` is n + 1 of them."""
import re

READ_AFTER_VALU = 2
SETTLED = 18  # a product of 32 x 32 x 16 has 16 passes


def _registers(token):
    """{(file, number)} of an operand like v7, a[0:15] or -v[2:3]."""
    m = re.match(r"-?\|?([va])(?:(\d+)|\[(\d+):(\d+)\])\|?$", token)
    if not m:
        return set()
    first, last = (int(m.group(2)),) * 2 if m.group(2) else (int(m.group(3)), int(m.group(4)))
    return {(m.group(1), r) for r in range(first, last + 1)}


class _Block:
    def __init__(self, label):
        self.label, self.code, self.target, self.falls, self.age = label, [], None, True, {}

    def end(self, target=None, falls=True):
        self.target, self.falls = target, falls
        return self


def _blocks(lines):
    out, block, in_asm = [], _Block(None), False
    for line in lines:
        if "ASMSTART" in line or "ASMEND" in line:
            in_asm = "ASMSTART" in line
            continue
        text = line.split(";")[0].strip()
        if text.endswith(":"):
            out.append(block.end())
            block = _Block(text[:-1])
        elif text and not text.startswith("."):
            block.code.append((text, in_asm))
            op = text.split()[0]
            if op.startswith(("s_branch", "s_cbranch")):
                out.append(block.end(text.split()[1], op != "s_branch"))
                block = _Block(None)
            elif op.startswith(("s_endpgm", "s_setpc")):
                out.append(block.end(falls=False))
                block = _Block(None)
    return out + [block.end()]


def _walk(block):
    """(products, faults, ages at the end).  An age is the wait states since a
    product wrote the accumulation register, up to SETTLED."""
    products, faults, age = 0, [], dict(block.age)
    written = {}        # register -> wait states since a vector instruction wrote it
    since_start = 0
    for text, in_asm in block.code:
        op, *args = [t for t in re.split(r"[\s,]+", text) if t]
        regs = [_registers(a) for a in args]
        states = 1
        if in_asm and op.startswith("v_mfma") and args[0].startswith("a"):
            products += 1
            reads = set().union(*regs[1:4])
            if since_start < READ_AFTER_VALU or any(written.get(r, READ_AFTER_VALU) < READ_AFTER_VALU for r in reads):
                faults.append(f"{block.label}: {text}")
            fresh = {r: 0 for r in regs[0]}
        else:
            if any(r in age for used in regs for r in used):
                faults.append(f"{block.label}: touched early: {text}")
            fresh = {}
            if op == "s_nop":
                states = int(args[0]) + 1
        written = {r: n + states for r, n in written.items() if n + states < READ_AFTER_VALU}
        age = {r: n + states for r, n in age.items() if n + states < SETTLED}
        age.update(fresh)
        since_start += states
        if op.startswith("v_") and not op.startswith("v_mfma") and regs:
            for r in regs[0] | (regs[1] if "swap" in op else set()):
                written[r] = 0
    return products, faults, age


def scan(lines):
    """(products written as assembly, faults) of a listing's lines."""
    blocks = _blocks(lines)
    at = {b.label: i for i, b in enumerate(blocks) if b.label}
    work = list(range(len(blocks)))
    while work:
        i = work.pop()
        out = _walk(blocks[i])[2]
        follow = ([at[blocks[i].target]] if blocks[i].target in at else []) + ([i + 1] if blocks[i].falls else [])
        for b in (blocks[j] for j in follow if j < len(blocks)):
            merged = {r: min(out.get(r, SETTLED), b.age.get(r, SETTLED)) for r in out.keys() | b.age.keys()}
            if merged != b.age:
                b.age = merged
                work.append(blocks.index(b))
    walks = [_walk(b) for b in blocks]
    return sum(w[0] for w in walks), [f for w in walks for f in w[1]]
