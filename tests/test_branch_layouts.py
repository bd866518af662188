"""Strides that the cross-attention calls take and refuse; the calls here are refused in the end, and no GPU is touched."""
import pytest

from paper_2607_04461_amd import flashbon as fb
from test_branch_validation import CROSS, CROSS_GRAD, at


def call(name, base, **change):
    args = dict(base, **change)
    status = getattr(fb.load(), "flashbon_op_" + name)(*args.values())
    return status, fb.load().flashbon_last_error().decode()


# batch 2, 3 rows of 64
APART = [(192, 64), (200, 64), (192 + 64, 72), (64, 128), (64, 192), (72, 136)]
TOGETHER = [(128, 64), (64, 64), (192, 56), (64, 120), (56, 128), (0, 64), (64, 0), (96, 64)]


@pytest.mark.parametrize("o_bs,o_rs", APART)
def test_rows_of_out_apart(o_bs, o_rs):
    """Batch rows behind each other, or side by side ([tq][batch][width]): refused here for lse alone, which lies on out."""
    status, why = call("cross_attention", CROSS, o_bs=o_bs, o_rs=o_rs, lse=at(5))
    assert status == fb.EINVAL and "overlap" in why, why


@pytest.mark.parametrize("o_bs,o_rs", TOGETHER)
def test_rows_of_out_together(o_bs, o_rs):
    status, why = call("cross_attention", CROSS, o_bs=o_bs, o_rs=o_rs, lse=at(5))
    assert status == fb.EINVAL and "apart" in why, why


@pytest.mark.parametrize("bs,rs", APART)
def test_rows_of_gradients_apart(bs, rs):
    """Refused here for the workspace alone."""
    assert call("cross_attention_grad", CROSS_GRAD, q_bs=bs, q_rs=rs, workspace=None)[0] == fb.ESHAPE
    # keys of 5 rows of 32, two prompts: rows of both prompts side by side
    assert call("cross_attention_grad", CROSS_GRAD, kv_bs=32, kv_rs=64, workspace=None)[0] == fb.ESHAPE


@pytest.mark.parametrize("bs,rs", TOGETHER)
def test_rows_of_gradients_together(bs, rs):
    status, why = call("cross_attention_grad", CROSS_GRAD, q_bs=bs, q_rs=rs, workspace=None)
    assert status == fb.EINVAL and "apart" in why, why


@pytest.mark.parametrize("kv_bs,kv_rs,away", [(32, 120, 64), (32, 128, 32), (64, 128, 16), (64, 120, 32), (160, 32, 32), (160, 32, 128),
                                              (312, 32, 160), (64, 128, 96)])
def test_keys_and_values_together(kv_bs, kv_rs, away):
    """Rows of dk and dv of which some share elements, or with no room between them for the others."""
    for first, second in ((0, away), (away, 0)):
        status, why = call("cross_attention_grad", CROSS_GRAD, kv_bs=kv_bs, kv_rs=kv_rs, dk=at(10) + 2 * first, dv=at(10) + 2 * second)
        assert status == fb.EINVAL and ("apart" in why or "overlap" in why), (status, why)


@pytest.mark.parametrize("batch,heads,tq,taken", [(7, 9, 1 << 24, False), (1, (1 << 24) - 1, 64, False), (3, 21, (1 << 24) - 63, False),
                                                  (8, 8, (1 << 24) - 64, True), (7, 9, (1 << 24) - 64, True), (1, (1 << 24) - 8, 64, True)])
def test_most_queries(batch, heads, tq, taken):
    """Launches take the pairs of batch row and head by eights: 2^24 blocks of 64 queries are 2^32 threads, one too many."""
    wide = heads * 8
    sizes = dict(batch=batch, heads=heads, kv_heads=1, head_dim=8, tq=tq, tk=1, q_bs=tq * wide, q_rs=wide, o_bs=tq * wide, o_rs=wide, n_kv=1)
    for name, base in (("cross_attention", CROSS), ("cross_attention_grad", CROSS_GRAD)):
        status, why = call(name, base, **sizes, out=None)
        assert status == (fb.EINVAL if taken else fb.ESHAPE), (name, why)       # refused for the missing out, or for its size
        assert ("required" in why) == taken


@pytest.mark.parametrize("table", ["kv_index", "kv_len", "lse"])
def test_tables_off_four_bytes(table):
    """Where the address is right, refused for the output or the workspace that the call lacks."""
    status, why = call("cross_attention", CROSS, **{table: CROSS[table] + 2, "out": CROSS["q"]})
    assert status == fb.EINVAL and "multiples" in why, why
    status, why = call("cross_attention_grad", CROSS_GRAD, **{table: CROSS_GRAD[table] + 2, "workspace": None})
    assert status == fb.EINVAL and "multiples" in why, why


def test_workspace_of_sizes_past_32_bits():
    """The binding's function refuses what the call's arguments would wrap, as the call does."""
    with pytest.raises(ValueError):
        fb.flashbon_op_layer_norm_grad_workspace(4096, 64, (1 << 32) + 4096)
    assert fb.flashbon_op_layer_norm_grad_workspace(4096, 64, 4096) > 0
