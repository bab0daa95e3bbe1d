"""The build refuses an attention gradient whose assembly statements lack wait
states: the scan finds planted hazards, and a fault of it leaves the library as it was."""
import os

import pytest

from paper_2608_21229_amd import build as rc_build
from paper_2608_21229_amd import wait_states

MFMA = [";;#ASMSTART", "v_mfma_f32_32x32x16_bf16 a[0:15], v[0:3], v[4:7], a[0:15]", ";;#ASMEND"]
CVT, OTHER = "v_cvt_pk_bf16_f32 v5, v8, v9", "ds_read_b128 v[20:23], v30"
READ = "v_accvgpr_read_b32 v1, a2"


@pytest.mark.parametrize("lines,faults", [
    ([CVT, "s_nop 1"] + MFMA, 0), ([CVT, OTHER, OTHER] + MFMA, 0), ([CVT, OTHER] + MFMA, 1), ([OTHER] + MFMA, 1),
    ([CVT, "s_nop 0"] + MFMA, 1), (["s_nop 1", "v_exp_f32 v9, v1"] + MFMA, 0),
    (["s_nop 1", "v_permlane32_swap_b32 v9, v6"] + MFMA, 1), (["s_nop 1", "v_accvgpr_write_b32 a5, 0", OTHER] + MFMA, 1),
    (["s_nop 1"] + MFMA + MFMA, 0), (["s_nop 1"] + MFMA + [READ], 1), (["s_nop 1"] + MFMA + ["s_nop 15", READ], 1),
    (["s_nop 1"] + MFMA + ["s_nop 15", "s_nop 1", READ], 0), (["s_nop 1"] + MFMA + ["v_accvgpr_read_b32 v1, a16"], 0),
    (["s_nop 1"] + MFMA + ["scratch_store_dwordx4 off, a[0:3], off"], 1),
    (["s_nop 1"] + MFMA + ["s_cbranch_scc1 y", "s_nop 15", "s_nop 15", "s_branch x", "y:", READ], 1),
    (["s_nop 1"] + MFMA + ["s_cbranch_scc1 y", "s_nop 15", "s_nop 15", "s_branch x", "y:", "s_nop 15", "s_nop 1", READ], 0),
    (["s_branch z", "y:", READ, "s_endpgm", "z:", "s_nop 1"] + MFMA + ["s_branch y"], 1)])
def test_scan(lines, faults):
    products, found = wait_states.scan(["x:"] + lines)
    assert products >= 1 and len(found) == faults, found


def test_a_listing_without_the_products_is_a_fault(tmp_path):
    name = tmp_path / "attn_bwd-hip-amdgcn-amd-amdhsa-gfx950.s"
    name.write_text("x:\ns_endpgm\n")
    assert "of 0 accumulator products" in rc_build._hazards("attn_bwd.hip", str(tmp_path))
    name.write_text("\n".join(["x:", CVT] + MFMA))
    assert "lack wait states" in rc_build._hazards("attn_bwd.hip", str(tmp_path))
    name.write_text("\n".join(["x:", CVT, "s_nop 1"] + MFMA))
    assert rc_build._hazards("attn_bwd.hip", str(tmp_path)) is None


def test_build_refuses_a_fault(monkeypatch, tmp_path):
    real, seen = wait_states.scan, []

    def planted(lines):
        products, faults = real(lines)
        seen.append(products)
        return products, faults + ["planted"]

    lib = tmp_path / "librefcache.so"
    lib.write_text("as it was")
    monkeypatch.setattr(rc_build, "LIB", str(lib))
    monkeypatch.setattr(rc_build, "SOURCES", ["attn_bwd.hip"])
    monkeypatch.setattr(wait_states, "scan", planted)
    with pytest.raises(RuntimeError, match="planted"):
        rc_build.build()
    assert seen and seen[0] >= 100, "the object's own listing was read"
    assert lib.read_text() == "as it was" and os.listdir(tmp_path) == ["librefcache.so"]
