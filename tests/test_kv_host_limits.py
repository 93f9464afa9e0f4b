"""Sizes past what one launch of the attention can hold are refused before any device is touched."""
import pytest

import paper_2603_25385_amd as G

P = 0x1000


def call(n_requests, kv_heads, T, heads, max_fresh=1):
    cache = G.make_kv_cache(P, P, P, P, 1 << 16, 16, kv_heads, 64)
    query = G.make_kv_attention(q=P, out=P, table=P, lengths=P, starts=P, ldq=heads * 64, ldo=heads * 64, table_width=8, n_requests=n_requests,
                                T=T, heads=heads, act_dtype=G.GLOWQ_F16, max_fresh=max_fresh, max_length=100, window=0, scale=0.125)
    return cache, query


# a workgroup for every 16 rows of a request's key/value head, 256 threads each, 2^32 threads a launch
@pytest.mark.parametrize("n,kv,heads,fresh", [(1 << 20, 16, 16, 1), (1 << 20, 1024, 1024, 1), (1 << 19, 64, 64, 1), (1 << 19, 64, 64, 17)])
def test_more_workgroups_than_a_launch_holds(n, kv, heads, fresh):
    cache, query = call(n, kv, 1 << 20, heads, fresh)
    for f in (lambda: G.glowq_kv_attention_workspace_bytes(cache, query), lambda: G.glowq_kv_attention(cache, query, P, 1 << 40)):
        with pytest.raises(G.GlowqError) as e:
            f()
        assert e.value.status == G.GLOWQ_ERR_SHAPE


@pytest.mark.parametrize("n,kv,heads,fresh", [(1 << 20, 8, 32, 1), (1 << 17, 64, 64, 1), (1, 1024, 1024, 1 << 20), (1 << 20, 15, 15, 1)])
def test_as_many_as_it_holds(n, kv, heads, fresh):
    assert G.glowq_kv_attention_workspace_bytes(*call(n, kv, 1 << 20, heads, fresh)) > 0
