"""The post-build check follows values through scratch memory and finds unpacked elements that nothing reads."""
import pytest

from paper_2607_21271_amd import isa_check

KERNEL = "_ZN3eqk19eql_scan_bwd_kernelILi1ELi16ELi1EEEvNS_8ScanArgsEi:"


def _scan(body):
    return [p[1] for p in isa_check.scan_lines([KERNEL] + body.strip("\n").split("\n"))]


def unpack(lo, hi, word):
    return ("\t;;#ASMSTART\n\tv_cvt_f32_f16_e32 v%d, v%d\n\tv_cvt_f32_f16_sdwa v%d, v%d dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:WORD_1\n"
            "\t;;#ASMEND\n" % (lo, word, hi, word))


@pytest.mark.parametrize("width,regs", [("", "v3"), ("x2", "v[2:3]"), ("x4", "v[1:4]")])
@pytest.mark.parametrize("where", ["", " offset:16"])
def test_a_spilled_result_stays_one(width, regs, where):
    """A convert of an fp32 result that came back from scratch memory."""
    body = "\tv_add_f32_e32 v3, v1, v2\n\tscratch_store_dword%s off, %s, off%s ; Folded Spill\n\tv_mov_b32_e32 v3, 0\n" \
           "\tscratch_load_dword%s %s, off, off%s ; Folded Reload\n\ts_waitcnt vmcnt(0)\n\tv_cvt_f32_f16_e32 v5, v3\n" % (
               width, regs, where, width, regs, where)
    assert _scan(body) == ["converted_source"]


def test_a_spilled_raw_word_is_converted():
    body = "\tv_add_f32_e32 v3, v1, v2\n\tbuffer_load_dword v4, v9, s[0:3], 0 offen\n\tscratch_store_dword off, v4, off offset:8\n" \
           "\tscratch_store_dword off, v3, off offset:12\n\tscratch_load_dword v3, off, off offset:8\n\tv_cvt_f32_f16_e32 v5, v3\n"
    assert _scan(body) == []
    # of another slot, of an unknown one, and after a branch nothing is known
    for body in ("\tv_add_f32_e32 v3, v1, v2\n\tscratch_store_dword off, v3, off\n\tscratch_load_dword v3, off, off offset:4\n\tv_cvt_f32_f16_e32 v5, v3\n",
                 "\tv_add_f32_e32 v3, v1, v2\n\tscratch_store_dword off, v3, off\n.LBB0_1:\n\tscratch_load_dword v3, off, off\n\tv_cvt_f32_f16_e32 v5, v3\n"):
        assert _scan(body) == []


LOST = unpack(38, 43, 1) + "\ts_and_b64 vcc, exec, s[28:29]\n\ts_cbranch_vccnz .LBB0_2\n\tv_mov_b32_e32 v37, v2\n.LBB0_2:\n" \
    + unpack(40, 43, 37) + "\tv_mov_b32_e32 v65, v43\n\tv_add_f32_e32 v1, v38, v40\n\tv_add_f32_e32 v1, v1, v65\n" \
    "\tglobal_store_dword v[2:3], v1, off\n\ts_endpgm\n"


def test_flags_an_element_whose_register_is_taken():
    """As it was emitted for the scan's gradients: x's element in v43, then dy's in v43, across a branch."""
    assert _scan(LOST) == ["lost_unpack"]


@pytest.mark.parametrize("reader", ["v_mov_b32_e32 v60, v43", "v_fmac_f32_e32 v43, v1, v2", "v_cmp_lt_f32_e32 vcc, 0, v43", "ds_write_b32 v9, v43",
                                    "scratch_store_dword off, v43, off offset:4", "v_cvt_pkrtz_f16_f32 v8, v[42:43], v2",
                                    "v_permlane32_swap_b32_e32 v43, v44", "v_add_f32_dpp v43, v1, v1 quad_perm:[1,0,3,2]", "s_swappc_b64 s[30:31], s[4:5]", "buffer_load_dwordx4 v43, s[0:3], 0 offen lds",
                                    "global_load_lds_dwordx4 v[42:43], off"])
def test_passes_where_it_is_read(reader):
    """On either way to where the register is written again."""
    assert _scan(LOST.replace("\ts_and_b64 vcc", "\t%s\n\ts_and_b64 vcc" % reader)) == []
    assert _scan(LOST.replace("\tv_mov_b32_e32 v37, v2\n", "\t%s\n" % reader)) == []


def test_passes_a_loop_that_reads_it_in_its_next_turn():
    body = "\tv_mov_b32_e32 v43, 0\n.LBB0_1:\n\tv_add_f32_e32 v9, v9, v43\n" + unpack(38, 43, 1) + "\tv_add_f32_e32 v9, v9, v38\n" \
        "\ts_cbranch_scc1 .LBB0_1\n\tglobal_store_dword v[2:3], v9, off\n\ts_endpgm\n"
    assert _scan(body) == []
    assert _scan(body.replace("s_cbranch_scc1 .LBB0_1", "s_nop 0")) == ["lost_unpack"]
