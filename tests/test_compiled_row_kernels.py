"""CPU test of the kernels of the linear cross entropy as they were compiled: those with one wave per SIMD keep their results in accumulation
registers that the compiler knows nothing of (csrc/wide_loop.hpp), also where the results are stored by csrc/xent_kernel.hpp.  Their
wait states are looked at with those of all kernels (test_compiled_kernels.py)."""
from tests.test_compiled_kernels import _registers, kernels  # noqa: F401


def test_accumulators_belong_to_the_assembly(kernels):  # noqa: F811
    wide = {name: code for name, code in kernels.items() if "11gemm_kernelINS_7XentCfg" in name and "Lb1EEELi" in name}
    assert len(wide) == 18                     # three tiles, three kinds of results, two types
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

