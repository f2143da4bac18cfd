"""Sizes whose launch would have more threads than a launch can have (2^32) are refused as unsupported, before it (no GPU: the addresses are never read)."""
import pytest

import paper_2007_12216_amd as rn
from test_host_decoder import A, UNSUPPORTED, attention, cache, code, rope


@pytest.mark.parametrize("head_dim,lanes", [(32, 8), (64, 8), (96, 16), (128, 16), (160, 32), (256, 32)])
@pytest.mark.parametrize("over", [0, 1, 2 ** 20])
def test_norm_and_rotation(head_dim, lanes, over):
    """A head takes `lanes` threads of workgroups of 256: 2^32 threads is one too many."""
    heads, kv = 12, 4
    strides = dict(q_stride=heads * head_dim, q_out_stride=heads * head_dim, k_stride=kv * head_dim, k_out_stride=kv * head_dim, v_stride=kv * head_dim)
    tokens = 2 ** 32 // lanes // (heads + kv) + over
    assert code(rn.rnswino_qk_norm_rope, rope(n_tokens=tokens, q_heads=heads, kv_heads=kv, head_dim=head_dim, rotary=0, **strides), A, A, A, A, A, A, A, A) == UNSUPPORTED
    tokens = -(-2 ** 32 // lanes // (heads + 2 * kv)) + over
    d = rope(n_tokens=tokens, q_heads=heads, kv_heads=kv, head_dim=head_dim, rotary=0, **strides)
    assert code(rn.rnswino_qk_norm_rope_cache4, d, A, A, A, A, A, A, A, A, A, cache(kv_heads=kv, head_dim=head_dim)) == UNSUPPORTED


@pytest.mark.parametrize("q_heads,kv_heads,requests,tokens,told", [(8, 8, 2 ** 21, 2 ** 21, 1), (8, 2, 2 ** 23, 2 ** 23, 1), (8, 2, 2 ** 23 + 5, 100, 0), (1, 1, 3, 2 ** 31 - 5, 0), (32, 32, 1, 2 ** 26 - 2, 0)])
@pytest.mark.parametrize("head_dim", [64, 96, 128, 256])
def test_attention(q_heads, kv_heads, requests, tokens, told, head_dim):
    """A tile of rows takes a workgroup of 256 for each key head and part of its positions: here there are 2^24 or more of those, by requests of one tile and by rows of few requests."""
    c = cache(kv_heads=kv_heads, head_dim=head_dim)
    d = attention(n_requests=requests, n_tokens=tokens, q_heads=q_heads, max_fresh=told, q_stride=q_heads * head_dim, out_stride=q_heads * head_dim)
    assert code(rn.rnswino_cache4_attention, c, d, A, A, A, A, A, A) == UNSUPPORTED
    assert rn.rnswino_cache4_attention_workspace_bytes(c, d) == 0


@pytest.mark.parametrize("page_size,width", [(16, 2 ** 27), (64, 2 ** 25), (4096, 2 ** 19), (4096, 2 ** 31 - 1)])
def test_attention_over_tables_of_more_positions_than_32_bits_number(page_size, width):
    """The kernels ask for the pages of some steps ahead of a request's last in 32-bit positions: with a length next to 2^31 those would be negative, in front of the table."""
    d = attention(table_width=width)
    assert code(rn.rnswino_cache4_attention, cache(page_size=page_size), d, A, A, A, A, A, A) == UNSUPPORTED
    assert rn.rnswino_cache4_attention_workspace_bytes(cache(page_size=page_size), d) == 0
    assert rn.rnswino_cache4_attention_workspace_bytes(cache(page_size=page_size), attention(table_width=width // 2)) > 0 or width == 2 ** 31 - 1
