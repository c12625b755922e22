"""Registers of the attention and vocabulary-loss kernels in the built library (CPU only): what the compiler notes
beside each kernel.  Their main loops hold running sums in nearly every register, and a register kept in memory there
is read back behind the loop's own loads."""
import re
import subprocess

import pytest

from paper_2607_28848_amd import build as pkg_build
from test_kernel_resources import READELF, _code_objects


@pytest.fixture(scope="module")
def notes(tmp_path_factory):
    out = {}
    for i, co in enumerate(_code_objects(pkg_build.LIB)):
        f = tmp_path_factory.mktemp("co") / ("%d.o" % i)
        f.write_bytes(co)
        text = subprocess.run([READELF, "--notes", str(f)], capture_output=True, text=True, check=True).stdout
        for m in re.finditer(r"\.group_segment_fixed_size: (\d+).*?\.name:\s+(\S+).*?\.vgpr_spill_count:\s+(\d+)", text, re.S):
            out[m.group(2)] = int(m.group(1)), int(m.group(3))
    return out


@pytest.mark.parametrize("name,most", [("attn_fwd_kernel", 0), ("attn_split_kernel", 0), ("attn_dk_kernel", 0),
                                       ("attn_dq_kernel", 8), ("attn_f32_", 0), ("vocab_logits_kernel", 32),
                                       ("vocab_grad_kernel", 32), ("vocab_f32_", 0)])
def test_registers(notes, name, most):
    """vocab: whole tiles of 256 rows take every register, and a few that only the prologue and epilogue use go to
    memory; dQ of heads of 128 reads its own rows' constants back once a tile."""
    found = {k: v for k, v in notes.items() if name in k}
    assert found and all(lds <= 160 * 1024 and spills <= most for lds, spills in found.values()), found
