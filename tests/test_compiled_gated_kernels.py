"""CPU test of the kernels of the gated feed-forward block as they were compiled: those with one wave per SIMD keep their results in accumulation
registers that the compiler knows nothing of (csrc/wide_loop.hpp), also where the results are stored by csrc/gated_kernel.hpp; and none of the new
kernels keeps anything in memory of its own (spilled registers)."""
from tests.test_compiled_kernels import _registers, kernels  # noqa: F401


def test_accumulators_belong_to_the_assembly(kernels):  # noqa: F811
    wide = {name: code for name, code in kernels.items() if "11gemm_kernelINS_8GatedCfg" in name and "Lb1EEELi" in name}
    assert len(wide) == 34                     # three tiles, five kinds of products, two types; and two kinds on the tile for two workgroups a unit
    for name, code in wide.items():
        cleared, read = [], set()
        for op, rest in code:
            operands = [o.strip() for o in rest.split(",")]
            touched = [o for o in operands if any(r[0] == "a" for r in _registers(o.split()[0] if o else o))]
            if not touched:
                continue
            if op == "v_accvgpr_write_b32":
                assert operands[1] == "0", (name, op, rest)
                cleared += _registers(operands[0])
            elif op == "v_accvgpr_read_b32":
                read |= _registers(operands[1])
            else:
                assert op.startswith("v_mfma_f32_16x16x32_") and touched == [operands[0], operands[3]] and operands[0] == operands[3], (name, op, rest)
        assert sorted(cleared) == [("a", i) for i in range(len(cleared))] and len(cleared) in (128, 256), name
        assert read == set(cleared), name
    assert sum("Li1ELb0ELi2ELb1EEELi" in name for name in wide) == 4


def test_nothing_is_spilled(kernels):  # noqa: F811
    ours = {name: code for name, code in kernels.items() if any(k in name for k in ("GatedCfg", "gated_few", "gated_pad", "gated_product", "gated_round", "9dw_of_few", "5adamwI", "grad_squares", "9grad_norm"))}
    assert len(ours) > 60
    for name, code in ours.items():
        assert not [op for op, _ in code if op.startswith("scratch_")], name
