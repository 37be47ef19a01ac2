"""The mx4 GEMM's accumulators stay in their registers from the first op of a tile to the last (no GPU).  The op is inline assembly that ties its result to its accumulator, so the
text of an op names one register twice whatever the compiler does around it: what would show is a copy, a store or a scratch access in between."""
import re

import pytest

OP = "v_mfma_scale_f32_16x16x128_f8f6f4"
ACCUMULATOR = re.compile(r"(?<![\w.])a(\d+|\[\d+:\d+\])(?!\w)")


def _kernels(text):
    """name -> instructions of each kernel of the GEMM"""
    found = {}
    for name, body in re.findall(r"^(_Z\S*mx4_gemm_kernel\S*):(.*?)^\.Lfunc_end", text, re.M | re.S):
        lines = (line.split(";")[0].strip() for line in body.splitlines())
        found[name] = [x for x in lines if x and x[0] != "." and not x.endswith(":")]
    return found


def _touched(ops):
    """(matrix ops, instructions between the first and the last that touch an accumulator or scratch memory without being one)"""
    at = [i for i, x in enumerate(ops) if x.startswith(OP)]
    between = ops[at[0]:at[-1] + 1]
    return len(at), [x for x in between if not x.startswith(OP) and (ACCUMULATOR.search(x) or "accvgpr" in x or x.startswith("scratch_"))]


def test_accumulators_are_not_touched_between_the_ops(assembly):
    kernels = _kernels(assembly["k_mx4"])
    tiles = {re.search(r"Li(\d+)ELi(\d+)E", n).groups() for n in kernels}
    assert tiles == {("8", "8"), ("8", "4"), ("4", "4"), ("4", "2")} and len(kernels) >= 12, sorted(kernels)
    for name, ops in kernels.items():
        am, bn = map(int, re.search(r"Li(\d+)ELi(\d+)E", name).groups())
        n, touched = _touched(ops)
        assert n >= am * bn * 4 and not touched, (name, n, touched[:5])


KERNEL = "_ZN15mx4_gemm_kernelILi8ELi8EE:\n\tv_accvgpr_write_b32 a0, 0\n\t%s a[0:3], v[2:5], v[6:9], a[0:3], v10, v11 op_sel_hi:[0,0,0]\n%s\t%s a[0:3], v[2:5], v[6:9], a[0:3], v10, v11\n" \
         "\tv_accvgpr_read_b32 v1, a0\n.Lfunc_end0:\n"


@pytest.mark.parametrize("line,seen", [
    ("\tds_read_b128 v[2:5], v40 offset:1024\n\ts_nop 1\n", False), ("\tv_mov_b32_e32 v2, 0xa1\n.LBB0_1:\n\ts_cbranch_scc1 .LBB0_1\n", False),
    ("\tv_accvgpr_mov_b32 a4, a0\n", True), ("\tv_accvgpr_read_b32 v1, a2\n", True), ("\tv_accvgpr_write_b32 a3, v1\n", True), ("\tscratch_store_dwordx2 off, v[0:1], off\n", True),
    ("\tbuffer_store_dwordx4 a[0:3], v1, s[0:3], 0 offen\n", True), ("\tv_mov_b32_e32 v1, a0\n", True)])
def test_the_check_finds_copies(line, seen):
    (ops,) = _kernels(KERNEL % (OP, line, OP)).values()
    n, touched = _touched(ops)
    assert n == 2 and bool(touched) == seen


def test_the_check_finds_a_copy_planted_in_the_built_kernels(assembly):
    """In front of every op, as the builtin's copies stand: each kernel is told."""
    text = re.sub(rf"^(\s*){OP}", rf"\1v_accvgpr_mov_b32 a255, a0\n\1{OP}", assembly["k_mx4"], flags=re.M)
    assert all(_touched(ops)[1] for ops in _kernels(text).values())
