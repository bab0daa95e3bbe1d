"""The attention gradient's accumulator products are written as single
statements of assembly, which the compiler's hazard recogniser does not see.
What they need is checked in the assembly that the build makes: at least two
wait states between a vector instruction and a matrix product that reads its
result (an LDS read is waited for by the compiler, as for any operand), and
the last products settled before anything else touches their accumulators."""
import re
import subprocess

from paper_2608_21229_amd import build as rc_build


def _registers(token, file="v"):
    m = re.match(file + r"\[(\d+):(\d+)\]$|" + file + r"(\d+)$", token)
    if not m:
        return set()
    if m.group(3) is not None:
        return {int(m.group(3))}
    return set(range(int(m.group(1)), int(m.group(2)) + 1))


SETTLED = 18  # wait states after a 16-pass product before another instruction may touch its result


def _blocks(lines):
    """Basic blocks in order: (label or None, [(text, in_asm)], targets, falls through)."""
    blocks, label, body, in_asm = [], None, [], False
    for line in lines:
        if "ASMSTART" in line or "ASMEND" in line:
            in_asm = "ASMSTART" in line
            continue
        text = line.split(";")[0].strip()
        if not text or (text.startswith(".") and not text.endswith(":")):
            continue
        if text.endswith(":"):
            blocks.append((label, body, None, True))
            label, body = text[:-1], []
            continue
        body.append((text, in_asm))
        op = text.split()[0]
        if op.startswith(("s_branch", "s_cbranch")):
            blocks.append((label, body, text.split()[1], op != "s_branch"))
            label, body = None, []
        elif op.startswith(("s_endpgm", "s_setpc")):
            blocks.append((label, body, None, False))
            label, body = None, []
    blocks.append((label, body, None, True))
    return blocks


def _walk(body, age):
    """(products, faults, ages at the end) of one block.  `age` holds, per
    accumulation register, the wait states since a product last wrote it."""
    products, faults = 0, []
    before = [("label", set())]  # (kind, written registers or wait states), newest last
    for text, in_asm in body:
        parts = [t.lstrip("-") for t in re.split(r"[\s,]+", text) if t]
        op, states = parts[0], 1
        if op.startswith("v_mfma") and in_asm and parts[1].startswith("a"):
            products += 1
            reads = _registers(parts[2]) | _registers(parts[3]) | {("a", r) for r in _registers(parts[4], "a")}
            waited = 0
            for kind, what in reversed(before):
                if waited >= 2:
                    break
                if kind == "label" or (kind == "valu" and what & reads):
                    faults.append(text)
                    break
                waited += what if kind == "nop" else 1
            before.append(("other", set()))
            age = {r: n + 1 for r, n in age.items() if n + 1 < SETTLED}
            age.update({r: 0 for r in _registers(parts[1], "a")})
            continue
        if any(r in age for t in parts[1:] for r in _registers(t, "a")):
            faults.append("touched early: " + text)
        if op == "s_nop":
            states = int(parts[1]) + 1
            before.append(("nop", states))
        elif op.startswith("v_") and not op.startswith("v_mfma"):
            both = _registers(parts[2]) if "swap" in op else set()
            before.append(("valu", _registers(parts[1]) | both | {("a", r) for r in _registers(parts[1], "a")}))
        else:
            before.append(("other", set()))
        age = {r: n + states for r, n in age.items() if n + states < SETTLED}
    return products, faults, age


def _scan(lines):
    """(accumulator products, faults) of an assembly listing, over every path:
    the youngest age of each register is carried along the branches."""
    blocks = _blocks(lines)
    at = {label: i for i, (label, *_) in enumerate(blocks) if label}
    entry = [{} for _ in blocks]
    work = list(range(len(blocks)))
    while work:
        i = work.pop()
        _, body, target, falls = blocks[i]
        _, _, out = _walk(body, entry[i])
        for j in ([at[target]] if target in at else []) + ([i + 1] if falls and i + 1 < len(blocks) else []):
            merged = {r: min(out.get(r, SETTLED), entry[j].get(r, SETTLED)) for r in out.keys() | entry[j].keys()}
            if merged != entry[j]:
                entry[j] = merged
                work.append(j)
    products, faults = 0, []
    for (_, body, _, _), age in zip(blocks, entry):
        n, bad, _ = _walk(body, age)
        products += n
        faults += bad
    return products, faults


def test_scan_sees_planted_hazards():
    mfma = [";;#ASMSTART", "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]", ";;#ASMEND"]
    cvt, other = "v_cvt_pk_bf16_f32 v5, v8, v9", "ds_read_b128 v[20:23], v30"
    assert _scan(["x:", cvt, "s_nop 1"] + mfma) == (1, [])
    assert _scan(["x:", cvt, other, other] + mfma) == (1, [])
    assert len(_scan(["x:", cvt, other] + mfma)[1]) == 1
    assert len(_scan(["x:", other] + mfma)[1]) == 1
    assert len(_scan(["x:", "v_accvgpr_write_b32 a5, 0", other] + mfma)[1]) == 1
    assert len(_scan(["x:", other, other] + mfma + ["v_accvgpr_read_b32 v1, a2"])[1]) == 1
    assert _scan(["x:", other, other] + mfma + ["s_nop 15", "s_nop 3", "v_accvgpr_read_b32 v1, a2"])[1] == []
    assert _scan(["x:", other, other] + mfma + ["v_accvgpr_read_b32 v1, a16"])[1] == []  # no product's result
    for touch in ("v_accvgpr_mov_b32 a20, a2", "scratch_store_dwordx4 off, a[0:3], off", "v_accvgpr_write_b32 a3, v1"):
        assert len(_scan(["x:", other, other] + mfma + [touch])[1]) == 1
    # along a branch: the loop's last product is read behind its exit
    loop = ["x:", other, other] + mfma + ["s_cbranch_scc1 y", "s_nop 15", "s_nop 15", "s_branch x", "y:"]
    assert len(_scan(loop + ["v_accvgpr_read_b32 v1, a2"])[1]) == 1
    assert _scan(loop + ["s_nop 15", "s_nop 1", "v_accvgpr_read_b32 v1, a2"])[1] == []


def test_accumulator_products_have_their_wait_states(tmp_path):
    out = str(tmp_path / "attn_bwd.s")
    r = subprocess.run(rc_build.compile_command("attn_bwd.hip", out, "--cuda-device-only", "-S"),
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    products, faults = _scan(open(out))
    assert products >= 100, "the accumulator products are not where the scan looks"
    assert not faults, faults[:5]
