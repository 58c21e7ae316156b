"""The learner's device code keeps to the hardware rules of this part, as
tests/test_isa_hygiene.py states them (CPU only)."""
import pytest

from paper_2207_07736_amd import build

rules = pytest.importorskip("test_isa_hygiene")


def test_device_code_has_no_packed_fp32_and_no_scalar_writes(tmp_path):
    text = open(build.asm(str(tmp_path / "out.s"), build.LEARN_SRC)).read()
    assert "v_mfma_f32_32x32x16_bf16" in text and "ds_read_b64_tr_b16" in text       # the assembly is the real kernels
    assert not rules.PACKED.findall(text) and not rules.SCALAR_WRITE.findall(text)
