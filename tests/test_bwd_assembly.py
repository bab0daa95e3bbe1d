"""The attention gradient's accumulator products are written as single
statements of assembly, which the compiler's hazard recogniser does not see.
What they need is checked in the assembly that the build makes: at least two
wait states between a vector instruction and a matrix product that reads its
result (an LDS read is waited for by the compiler, as for any operand), and
the last products settled before their accumulators are read."""
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


def _scan(lines):
    """(accumulator products, faults) of an assembly listing."""
    products, faults = 0, []
    before = []           # (kind, written registers or wait states), newest last
    since_product = None  # wait states since the last accumulator product
    in_asm = False
    for line in lines:
        if "ASMSTART" in line or "ASMEND" in line:
            in_asm = "ASMSTART" in line
            continue
        text = line.split(";")[0].strip()
        if not text or (text.startswith(".") and not text.endswith(":")):
            continue
        if text.endswith(":"):
            before = [("label", set())]
            continue
        parts = [t for t in re.split(r"[\s,]+", text) if t]
        op = parts[0]
        if op.startswith("v_mfma") and in_asm and parts[1].startswith("a"):
            products += 1
            reads, states = _registers(parts[2]) | _registers(parts[3]), 0
            for kind, what in reversed(before):
                if states >= 2:
                    break
                if kind == "label" or (kind == "valu" and what & reads):
                    faults.append(text)
                    break
                states += what if kind == "nop" else 1
            since_product = 0
            before.append(("other", set()))
            continue
        if op.startswith("v_accvgpr_read") and since_product is not None and since_product < 18:
            faults.append("read early: " + text)
        if op == "s_nop":
            before.append(("nop", int(parts[1]) + 1))
        elif op.startswith("v_") and not op.startswith("v_mfma"):
            both = _registers(parts[2]) if "swap" in op else set()
            before.append(("valu", _registers(parts[1]) | both))
        else:
            before.append(("other", set()))
        if since_product is not None:
            since_product += before[-1][1] if op == "s_nop" else 1
    return products, faults


def test_scan_sees_planted_hazards():
    mfma = [";;#ASMSTART", "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]", ";;#ASMEND"]
    cvt, other = "v_cvt_pk_bf16_f32 v5, v8, v9", "ds_read_b128 v[20:23], v30"
    assert _scan(["x:", cvt, "s_nop 1"] + mfma) == (1, [])
    assert _scan(["x:", cvt, other, other] + mfma) == (1, [])
    assert len(_scan(["x:", cvt, other] + mfma)[1]) == 1
    assert len(_scan(["x:", other] + mfma)[1]) == 1
    assert len(_scan(["x:", other, other] + mfma + ["v_accvgpr_read_b32 v1, a2"])[1]) == 1
    assert _scan(["x:", other, other] + mfma + ["s_nop 15", "s_nop 3", "v_accvgpr_read_b32 v1, a2"])[1] == []


def test_accumulator_products_have_their_wait_states(tmp_path):
    out = str(tmp_path / "attn_bwd.s")
    r = subprocess.run(rc_build.compile_command("attn_bwd.hip", out, "--cuda-device-only", "-S"),
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    products, faults = _scan(open(out))
    assert products >= 100, "the accumulator products are not where the scan looks"
    assert not faults, faults[:5]
