"""What the compiler made of the kernels of linear attention and of the root-mean-square normalization: they keep all their registers (a reload from scratch
memory waits for the rows that are on their way)."""
import pytest

from test_kernel_resources import kernel_notes


@pytest.mark.parametrize("kernel,variants", [("sweep_kernel", 6), ("back_kernel", 17), ("states_kernel", 3), ("scan_kernel", 3), ("step_kernel", 3),
                                             ("3rms10fwd_kernel", 32), ("3rms10bwd_kernel", 32)])
def test_no_scratch(tmp_path, kernel, variants):
    notes = [n for n in kernel_notes(tmp_path) if kernel in n[0]]
    assert len(notes) >= variants
    assert not [n for n in notes if n[1] or n[2]]
