"""The cases of appending to the cache, of attention over it and of decoding once more, with comparisons that a NaN cannot pass: hidden places of the
pools, and cache and workspace before their first use, hold NaN there, and a NaN is neither above a bound nor the larger of two errors."""
import pytest

import test_gpu_decode as decode
import test_gpu_generate as generate
from helpers import rel_fro_of_numbers, within
from test_gpu_decode import (  # noqa: F401  (run here with the comparisons below)
    test_append, test_append_at_far_positions, test_append_of_many_rows, test_append_prompts_and_single_tokens, test_append_strides,
    test_attention_in_pairs_of_tiles, test_attention_in_tiles_of_rows, test_attention_in_tiles_over_long_sequences, test_attention_lengths,
    test_attention_of_drafts_over_long_sequences, test_attention_of_extreme_scores, test_attention_of_rows_that_share_sequences,
    test_attention_over_long_sequences_of_few_rows, test_attention_strides, test_attention_without_pages, test_cache_beyond_32_bits, test_pages_that_sequences_share)
from test_gpu_generate import test_generation_as_it_is_used, test_prompt_then_single_tokens_give_the_oracles_logits  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def numbers_only(monkeypatch):
    monkeypatch.setattr(decode, "_close", within)
    monkeypatch.setattr(generate, "rel_fro", rel_fro_of_numbers)
