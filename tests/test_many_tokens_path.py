"""Launches of more threads than a dimension of a grid counts: the calls of the GPU test that reach one."""
import paged_choice as choice
import test_gpu_many_tokens as many


def test_the_call_of_many_heads_is_units_of_more_threads_than_32_bits_count():
    path = choice.path(many.HEADS, many.HEADS, [(1, 1)] * many.SEQUENCES, many.HINTS, 8, many.TABLE)
    assert path == "units 4"
    assert (many.SEQUENCES // 32 + many.SEQUENCES) * many.HEADS * 4 * 64 >= 1 << 32


def test_tokens_beyond_a_dimension():
    assert choice.parts(many.TOKENS, 1) == 1 and choice.parts(many.TOKENS, 2) == 1
    assert many.TOKENS * 64 >= 1 << 32
