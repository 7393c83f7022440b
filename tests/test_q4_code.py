"""What the compiler makes of the attention over the 4-bit cache and of the sampled fill: the attention keeps everything in registers, and so does what
every row of the fill runs (only the search of a whole row, for which it is rare, saves registers in memory)."""
import pytest

from tests.test_attention_code import _compiled, _kernels


@pytest.fixture(scope="module")
def attention(tmp_path_factory):
    return _compiled(tmp_path_factory, "fc_q4_attn.hip")


def test_attention_keeps_its_registers(attention):
    found = _kernels(attention, "k_q4_attn") + _kernels(attention, "k_q4_merge")
    assert len(found) == 24
    for name, code, _, scratch in found:
        assert scratch == 0 and not any(op.startswith(("scratch_", "v_accvgpr")) for op, _, _ in code), (name, scratch)


def test_queries_are_multiplied_as_they_are(attention):
    """Scores by bfloat16 products, 16 (heads of 64: 8) of them to a tile and row tile of bf16 rows, three times as many of fp32 ones; no instruction
    converts 32 values at once (their results may overlap their sources)."""
    for name, code, _, _ in _kernels(attention, "k_q4_attn"):
        products = sum(op == "v_mfma_f32_16x16x32_bf16" for op, _, _ in code)
        rows, parts = (2 if "ELi2ELi" in name else 1), (3 if "k_q4_attnIf" in name else 1)
        assert products == (16 if "Li128E" in name else 8) * rows * parts, (name, products)
        assert not any("pk16" in op or "pk32" in op or "f8f6f4" in op for op, _, _ in code), name


def test_every_row_of_a_fill_keeps_its_registers(tmp_path_factory):
    asm = _compiled(tmp_path_factory, "fc_sample.hip")
    found = _kernels(asm, "k_sample_pick") + _kernels(asm, "k_sample_bins") + _kernels(asm, "select_few") + _kernels(asm, "select_one_each")
    assert len(found) == 2 + 6 + 2
    for name, code, _, _ in found:
        assert not any(op.startswith("scratch_") for op, _, _ in code), name
