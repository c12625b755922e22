"""Registers of the rotation's and the distillation's kernels in the built library (CPU only): none keeps one in memory."""
import pytest

from test_operator_resources import notes  # noqa: F401  (a fixture)


@pytest.mark.parametrize("name,forms", [("rope_fwd_kernel", 8), ("rope_bwd_kernel", 8), ("rope_weight_kernel", 2), ("vocab_entry_kernel", 2),
                                        ("vocab_fold_kernel", 4), ("vocab_kd_finish_kernel", 2), ("vocab_finish_kernel", 2),
                                        ("attn_join_kernel", 2), ("attn_f32_grad_kernel", 2)])
def test_registers(notes, name, forms):  # noqa: F811
    found = {k: v for k, v in notes.items() if name in k}
    assert len(found) == forms and all(lds <= 64 * 1024 and spills == 0 for lds, spills in found.values()), found
