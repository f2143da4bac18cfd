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
