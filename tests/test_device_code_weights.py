"""The rows of queries that the attention weights bring straight into LDS: waited for before every barrier (CPU only:
the library's gfx950 code, disassembled)."""
import pytest

from test_device_code import OBJDUMP, functions, unwaited


@pytest.mark.skipif(OBJDUMP is None, reason="needs llvm-objdump")
def test_rows_are_waited_for_before_the_barrier(tmp_path):
    kernels = functions(tmp_path, "weights_turn_kernel")
    kernels = {n: c for n, c in kernels.items() if any("load_lds" in op for _, op, _ in c)}
    assert len(kernels) == 8        # bf16 queries: two head sizes, plain and 4-bit keys, one or more stages of rows
    for name, code in kernels.items():
        assert all(t is not None for _, op, t in code if op.startswith(("s_branch", "s_cbranch")))
        assert not any(op.startswith(("s_setpc", "s_swappc")) for _, op, _ in code)
        assert not unwaited(code), name
