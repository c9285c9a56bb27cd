"""Sizes of more than 32 bits in the binding of layer norm, rotary positions and the gated feed-forward block: refused, or what they mean -
never the low 32 bits of them.  Host only (tensors without storage)."""
import pytest

from paper_2511_20390_amd import binding as b

FAR = (1 << 32) + 4                  # low 32 bits: four


def _meta(*shape, dtype="bfloat16"):
    import torch
    return torch.empty(*shape, dtype=getattr(torch, dtype), device="meta")


def _refused(call):
    with pytest.raises(b.FreeError) as e:
        call()
    assert e.value.status == b.FREE_ERR_LIMIT


def test_tensors_of_more_rows():
    rows, pos = _meta(FAR, 2), _meta(1, 1, dtype="int32")
    for call in (lambda: b.op_layer_norm(rows), lambda: b.op_layer_norm_backward(rows, rows),
                 lambda: b.op_rope_axes(rows, pos, 1, 2, [2]),
                 lambda: b.op_rope_axes(_meta(4, 2), _meta(FAR, 1, dtype="int32"), 1, 2, [2]),
                 lambda: b.op_gated_ffn(rows, _meta(2, 2), _meta(2, 1)),
                 lambda: b.op_gated_ffn_backward(rows, rows, _meta(2, 2), _meta(2, 1), None),
                 lambda: b.op_gated_ffn(_meta(1, FAR), _meta(2, FAR), _meta(FAR, 1)),
                 lambda: b.op_gated_ffn(_meta(1, 2), _meta(2 * FAR, 2), _meta(2, FAR))):
        _refused(call)


def test_arguments_of_more_bits():
    _refused(lambda: b.op_rope_axes(_meta(4, 64), _meta(4, 1, dtype="int32"), 1, 64, [(1 << 32) + 64]))
    _refused(lambda: b.op_rope_axes(_meta(4, 64), _meta(4, 1, dtype="int32"), 1, 64, [-(1 << 32) + 64]))
    for call in (lambda: b.layer_norm_backward_workspace_bytes(FAR, 64), lambda: b.layer_norm_backward_workspace_bytes(8, FAR),
                 lambda: b.gated_ffn_saved_bytes(FAR, 64, 64, "bf16"), lambda: b.gated_ffn_saved_bytes(8, 64, FAR, "fp32"),
                 lambda: b.gated_ffn_workspace_bytes(FAR, 64, 64, "fp32"), lambda: b.gated_ffn_workspace_bytes(8, FAR, 64, "bf16", True)):
        _refused(call)


def test_rows_of_more_values():
    """A row may have more than 2^32 values where heads and their widths are numbers of 32 bits (what fails next: it has no storage)."""
    with pytest.raises(b.FreeError) as e:
        b.op_rope_axes(_meta(1, 1 << 32), _meta(1, 1, dtype="int32"), 1 << 25, 128, [128])
    assert e.value.status == b.FREE_ERR_NULL
    _refused(lambda: b.op_rope_axes(_meta(1, FAR + 60), _meta(1, 1, dtype="int32"), 1, FAR + 60, [64]))


def test_strides_of_more_bits():
    """Vectors of a sample four billion values behind those of the one before."""
    import types
    t = types.SimpleNamespace(is_cuda=True, dtype=_meta(1, dtype="float32").dtype, shape=(2, 64), stride=lambda axis: (FAR + 60, 1)[axis],
                              data_ptr=lambda: 4096)
    _refused(lambda: b._vectors(t, "weight", 2, 64))
    t.stride = lambda axis: (64, 1)[axis]
    assert b._vectors(t, "weight", 2, 64) == (4096, 64)


@pytest.mark.parametrize("rows", [8, 9, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, FAR, 1 << 63])
def test_any_number_of_rows_per_sample(rows):
    """rows_per_sample >= M is one sample: (1 << 32) + 1 must not be taken as samples of one row, whose weights lie behind the given ones."""
    assert b._norm_rows(_meta(8, 64), rows) == (8, 64, 8, 1)
    assert b.layer_norm_backward_workspace_bytes(8, 64, rows) == b.layer_norm_backward_workspace_bytes(8, 64)
    assert b._norm_rows(_meta(0, 64), rows) == (0, 64, 1, 1)
    assert b._norm_rows(_meta(8, 64), 3) == (8, 64, 3, 3)


@pytest.mark.parametrize("mode,step,size", [("bf16", 8, 2), ("fp32", 64, 4)])
def test_which_widths_are_copied(mode, step, size):
    """Room for padded copies of the weights is asked for where a width is no multiple of 8 (bf16) or 64 (fp32), and nowhere else."""
    for D, F in ((1152, 2688), (1152, 2688 + step), (1152 + step, 2688), (1152 + step, 2688 + 3 * step)):
        copies = 3 * D * F * size
        for backward in (False, True):
            room = lambda *widths: b.gated_ffn_workspace_bytes(40, *widths, mode, backward)
            least = 40 * F * size * (2 if backward else 1)                   # h, or its two gradients
            assert room(D, F) < least + copies
            for widths in ((D, F + step // 2), (D + 1, F), (D + step // 2, F - 1)):
                assert room(*widths) > least + copies * (1.9 if backward else 0.99)
