"""The build's check that results of multiplies are waited for on every path: what it has to find.  No compiler, no GPU."""
import pytest

from paper_2605_14305_amd import build as b

MUL = "v_mfma_f32_16x16x32_bf16 v[0:3], v[100:103], v[104:107], v[0:3]"
OTHER = "v_mfma_f32_16x16x32_bf16 v[4:7], v[100:103], v[104:107], v[4:7]"


def _kernel(*body):
    return ["_ZN3fef12_GLOBAL__N_115mx4_tile_kernelILi1EE:", *[x if x.startswith(".") else "\t" + x for x in body], "\ts_endpgm", ".Lfunc_end0:"]


@pytest.mark.parametrize("body", [
    [MUL, "s_nop 7", "v_mov_b32_e32 v20, v0"],
    [MUL, MUL, OTHER, "s_nop 7", "v_mov_b32_e32 v20, v0"],
    [MUL, "v_mov_b32_e32 v20, v21", "ds_write_b128 v30, v[4:7]", "s_nop 5", "ds_write_b128 v30, v[0:3]"],
    [".LBB0_1:", MUL, "s_cbranch_scc1 .LBB0_1", "s_nop 6", "v_mov_b32_e32 v20, v1"],
    ["s_branch .LBB0_1", "v_mov_b32_e32 v20, v0", ".LBB0_1:", MUL],
])
def test_accepts(body):
    b.check_results(_kernel(*body), verbose=False)


@pytest.mark.parametrize("body", [
    [MUL, "v_mov_b32_e32 v20, v0"],
    [MUL, "s_nop 6", "v_mov_b32_e32 v20, v3"],
    [MUL, "s_nop 3", "v_mov_b32_e32 v2, 0"],                      # overwritten before it is there
    [MUL, OTHER, "global_store_dwordx4 v30, v[0:3], s[0:1]"],
    # the short way past a block, the way that the compiler does not look at
    [MUL, "s_cbranch_vccnz .LBB0_2", OTHER, "s_nop 7", ".LBB0_2:", "v_mov_b64_e32 v[20:21], v[2:3]"],
    [".LBB0_1:", "ds_write_b128 v30, v[0:3]", MUL, "s_cbranch_scc1 .LBB0_1"],
])
def test_finds(body):
    with pytest.raises(RuntimeError, match="wait states behind"):
        b.check_results(_kernel(*body), verbose=False)


def test_wants_kernels_and_multiplies():
    with pytest.raises(RuntimeError, match="no kernel"):
        b.check_results(["_ZN3fef5otherE:", ".Lfunc_end0:"], verbose=False)
    with pytest.raises(RuntimeError, match="no multiply"):
        b.check_results(_kernel("v_mov_b32_e32 v1, v2"), verbose=False)
