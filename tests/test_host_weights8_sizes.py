"""Workspace of contexts with weights in 8 bits."""
import pytest


@pytest.mark.parametrize("kind", [1, 3])
def test_rows_in_8_bits_take_the_place_of_those_in_bf16(kind):
    """Beside the 8-bit cache, whose layers hand on the same sums in fp32: operands in 8 bits instead of bf16 are at most 0.51 of the bytes; the linear maps' own part is below 2 MB."""
    from paper_2511_13587_amd import binding as vb
    from paper_2511_13587_amd import synth
    for shape in (synth.SEVEN_B, synth.XL_TREE, synth.B_SHAPE):
        _, same, _ = vb.vvs_query_sizes(vb.make_config(shape, cache_kind=vb.VVS_CACHE_E4M3))
        _, held8, _ = vb.vvs_query_sizes(vb.make_config(shape, cache_kind=vb.VVS_CACHE_E4M3, weight_kind=kind))
        chunk = min(512, max(64, 4096 // shape.n_rows // 32 * 32), shape.prefix_len + shape.grid - 1)       # tokens per row of a prefill's passes
        operands = 2 * shape.n_rows * chunk * (shape.d_model + shape.d_ff)                                  # bytes in bf16
        assert held8 <= same - 0.48 * operands + (2 << 20), shape.name
