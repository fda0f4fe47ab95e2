"""The generated code of the kernels for ragged batches (no GPU): nothing goes through scratch memory."""
import pytest

from tests.test_few_row_code import _kernels


@pytest.mark.parametrize("source,name,count", [("attention_masked.hip", "masked_attn_tile_kernel", 20), ("attention_masked.hip", "masked_attn_rows_kernel", 5),
                                               ("attention_masked.hip", "masked_attn_order_kernel", 1),
                                               ("attention_masked.hip", "masked_attn_f32_kernel", 2), ("attention_masked.hip", "masked_attn_merge_kernel", 5),
                                               ("batch_rows.hip", "norm_rotary_kernel", 6), ("batch_rows.hip", "rotary_move_kernel", 3),
                                               ("batch_rows.hip", "batch_map_kernel", 1)])
def test_no_scratch(tmp_path, source, name, count):
    kernels = _kernels(tmp_path, source, name)
    assert len(kernels) == count
    assert all(scratch == 0 for _, scratch in kernels.values())
