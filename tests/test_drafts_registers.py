"""The kernels of a step of drafted tokens and of the rotation keep what they work on in registers, as the other serving
kernels do (checked on the CPU, from the compiler's own figures)."""
import pytest

from test_device_code_registers import test_no_kernel_uses_scratch_memory as check


@pytest.mark.parametrize("name", ["drafts", "rotate"])
def test_no_kernel_uses_scratch_memory(name, tmp_path):
    check(name, tmp_path)
