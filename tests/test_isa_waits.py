"""Wait states that the instruction set leaves to the program: the check of the library's code, on short sequences and on the library itself."""
import pytest

from paper_2504_20039_amd import check_isa

LOAD = "global_load_lds_dwordx4 v1, s[8:9]"


@pytest.mark.parametrize("between,missing", [([], 1), (["s_nop 0"], 0), (["v_add_u32_e32 v2, s3, v4"], 0)])
@pytest.mark.parametrize("load", [LOAD, "global_load_lds_dwordx4 v[2:3], off nt", "buffer_load_dwordx4 v1, s[4:7], 0 offen lds"])
@pytest.mark.parametrize("write", ["s_mov_b32 m0, s33", "s_add_i32 m0, s4, 0x400"])
def test_a_load_behind_a_write_of_m0(between, missing, load, write):
    found = check_isa.missing_waits(["_Z1kv:", write, *between, load])
    assert len(found) == missing and all("_Z1kv" in x for x in found)


def test_loads_that_do_not_read_m0():
    assert not check_isa.missing_waits(["s_mov_b32 m0, s33", "global_load_dwordx4 v[0:3], v1, s[8:9]"])
    assert not check_isa.missing_waits(["s_mov_b32 s0, m0", LOAD])
    assert not check_isa.missing_waits(["s_mov_b32 m0, s33 // 000000002EF4: BEFC0021", "s_endpgm", "0000000000001900 <_Z1kv>:", LOAD])


@pytest.mark.parametrize("write", ["v_readlane_b32 s9, v252, 10", "v_readfirstlane_b32 s8, v1", "v_cmp_eq_u32_e64 s[8:9], v1, v2", "v_add_co_u32_e64 v1, s[8:9], v2, v3",
                                   "v_mad_u64_u32 v[2:3], s[8:9], v4, v5, 0"])
@pytest.mark.parametrize("between,missing", [([], 1), (["s_nop 3"], 1), (["s_nop 4"], 0), (["s_mov_b32 m0, s3", "s_nop 0"], 1), (["s_waitcnt vmcnt(7)"] * 4, 1),
                                             (["v_add_u32_e32 v2, v3, v4"] * 5, 0), (["s_nop 1", "s_nop 1", "s_nop 0"], 0)])
def test_a_base_that_a_vector_instruction_wrote(write, between, missing):
    assert len(check_isa.missing_waits(["_Z1kv:", write, *between, LOAD])) == missing
    # of another register, or written once more by a scalar instruction, it is none
    assert not check_isa.missing_waits([write, *between, "s_nop 0", "global_load_lds_dwordx4 v1, s[10:11]"])
    assert not check_isa.missing_waits([write, *between, "s_mov_b64 s[8:9], s[4:5]", LOAD])
    assert not check_isa.missing_waits([write, *between, "_Z2k2v:", LOAD])


def test_the_library_keeps_them():
    import paper_2504_20039_amd as aj
    lines = check_isa.disassemble(aj.library_path())
    assert sum("global_load_lds_dwordx4" in x for x in lines) > 1000      # (the code was found)
    assert not check_isa.missing_waits(lines)
