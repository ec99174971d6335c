"""Refusals and limits of the serving operators' C ABI and of their functions
on tensors, on the CPU, beside those of test_serve_abi_cpu.py."""
import pytest

import paper_2601_18999_amd as K
from test_serve_abi_cpu import P, _names, _refused, attention, cache, store, tables


BAD_BASES = [dict(d_base=3 * P), dict(d_held=5 * P, d_held_out=P)]


@pytest.mark.parametrize("bad", BAD_BASES, ids=_names(BAD_BASES))
def test_a_base_that_the_call_would_overwrite_is_refused(bad):
    _refused(lambda: K.kvr_block_tables(tables(**bad), P, 1 << 20))


def test_more_workgroups_than_a_launch_holds_are_refused():
    # a workgroup has 256 threads, a launch fewer than 2^32
    most = 1 << 20
    K.kvr_attention_workspace(cache(kv_heads=15), attention(num_tokens=most, num_requests=most, num_groups=0, heads=15))
    for kv, heads in ((16, 16), (16, 64), (1024, 1024)):
        big = (cache(kv_heads=kv), attention(num_tokens=most, num_requests=most, num_groups=0, heads=heads))
        _refused(lambda: K.kvr_attention_workspace(*big))
        _refused(lambda: K.kvr_shared_attention(*big, P, 1 << 60))


@pytest.mark.parametrize("groups", [0, 1])
def test_the_workspace_of_one_long_prompt_does_not_grow_with_it(groups):
    # its rows have partial results only in as many items as the device holds at once
    def size(tokens):
        return K.kvr_attention_workspace(cache(kv_heads=8), attention(num_tokens=tokens, num_requests=1,
                                                                      num_groups=groups, heads=32))
    assert size(9216) < 80 << 20 and size(131072) < size(9216) + (8 << 20)


def test_more_tokens_than_a_store_counts_are_refused():
    # chunks of 8 elements of all tokens: at most 2^31 - 257
    for kv, dim, tokens in ((1, 64, (1 << 28) - 32), (8, 128, (1 << 24) - 2), (1024, 256, 1 << 16)):
        assert tokens * kv * dim // 8 > (1 << 31) - 257
        _refused(lambda: K.kvr_cache_store(cache(kv_heads=kv, dim=dim), store(num_tokens=tokens)))
