"""The build's check that the losses' matrix products keep their distance from what
writes their operands, on made-up disassembly."""
import pytest

from paper_2407_17353_amd import build

MFMA = "v_mfma_f32_16x16x32_f16 a[0:3], v[4:7], v[8:11], a[0:3]"


@pytest.mark.parametrize("before,sound", [
    (["v_mov_b32 v5, v1"], False), (["v_mov_b32 v5, v1", "s_nop 0"], False), (["v_mov_b32 v5, v1", "s_nop 1"], True),
    (["v_mov_b32 v5, v1", "s_add_i32 s1, s1, 4", "v_add_u32 v1, v1, v2"], True), (["v_mov_b32 v12, v1"], True),
    (["v_cvt_scalef32_pk_f16_fp8 v11, v1, 1.0"], False), (["ds_read_b128 v[4:7], v1"], True), (["v_cmp_lt_u32 vcc, v4, v1"], True)])
def test_products_keep_their_distance(before, sound):
    assert (build.product_distance_violations([*before, MFMA]) == []) == sound
    if sound:
        assert build.check_functions("/x/loss_logits.hip.o", {"k": [*before, MFMA]}) == 1
    else:
        with pytest.raises(RuntimeError, match="too soon"):
            build.check_functions("/x/loss_logits.hip.o", {"k": [*before, MFMA]})
