"""The output head's part of the C ABI that needs no device, and its device code's
hygiene (the same rules as the rest of the library's)."""
import re

import pytest

from paper_2207_07736_amd import build

PACKED = re.compile(r"^\s*v_pk_(fma|mul|add)_f32\b", re.M)
SCALAR_WRITE = re.compile(r"^\s*s_(store|buffer_store|scratch_store|atomic|buffer_atomic|dcache_wb|dcache_discard)\w*",
                          re.M)


@pytest.mark.parametrize("rows,vocab", [(0, 10), ((1 << 30) + 1, 10), (10, 0), (10, (1 << 20) + 1), (2 ** 32 - 1, 2 ** 32 - 1)])
def test_create_rejects_bad_sizes(rows, vocab):
    import paper_2207_07736_amd as p
    with pytest.raises(p.RlsimError) as e:
        p.rlsim_head_create(rows, vocab)
    assert e.value.code == p.RLSIM_EINVAL
    assert p.rlsim_head_last_error(None)


def test_null_handles():
    import paper_2207_07736_amd as p
    assert p.lib.rlsim_head_create(1, 1, None, None) == p.RLSIM_EINVAL
    assert p.lib.rlsim_head_sample(None, None) == p.RLSIM_EINVAL
    assert p.lib.rlsim_head_distill(None, None) == p.RLSIM_EINVAL
    assert p.lib.rlsim_head_destroy(None) == p.RLSIM_OK
    p.rlsim_head_destroy(None)


def test_device_code_has_no_packed_fp32_and_no_scalar_writes(tmp_path):
    text = open(build.asm(str(tmp_path / "head.s"), build.HEAD_SRC)).read()
    assert "k_sample" in text and "k_distill" in text
    assert not PACKED.findall(text), PACKED.findall(text)[:5]
    assert not SCALAR_WRITE.findall(text), SCALAR_WRITE.findall(text)[:5]
