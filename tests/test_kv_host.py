"""Refusals of the serving operators: documented status codes, before any device is touched."""
import pytest

import paper_2603_25385_amd as G

P = 0x1000


def cache(**kw):
    f = dict(k_codes=P, v_codes=P, k_scales=P, v_scales=P, n_blocks=10, block_tokens=32, kv_heads=4, head_dim=128)
    f.update(kw)
    return G.make_kv_cache(**f)


def query(**kw):
    f = dict(q=P, out=P, table=P, lengths=P, starts=P, ldq=1024, ldo=1024, table_width=8, n_requests=3, T=12, heads=8,
             act_dtype=G.GLOWQ_F16, max_fresh=4, max_length=200, window=0, scale=0.1)
    f.update(kw)
    return G.make_kv_attention(**f)


def step(**kw):
    f = dict(cached=P, fresh=P, free_blocks=P, table=P, lengths=P, starts=P, slots=P, positions=P, taken=P, n_requests=3, n_free=4,
             table_width=8, max_tokens=12, block_tokens=32)
    f.update(kw)
    return G.make_kv_step(**f)


def status(call):
    with pytest.raises(G.GlowqError) as e:
        call()
    return e.value.status


NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED, WS = (G.GLOWQ_ERR_NULL, G.GLOWQ_ERR_SHAPE, G.GLOWQ_ERR_ALIGN, G.GLOWQ_ERR_DTYPE,
                                              G.GLOWQ_ERR_UNSUPPORTED, G.GLOWQ_ERR_WORKSPACE)
BAD_CACHES = [(dict(n_blocks=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=1025), SHAPE), (dict(head_dim=0), SHAPE),
              (dict(block_tokens=0), SHAPE), (dict(block_tokens=-16), SHAPE), (dict(n_blocks=1 << 28), SHAPE),
              (dict(block_tokens=48), UNSUPPORTED), (dict(block_tokens=256), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
              (dict(head_dim=256), UNSUPPORTED)]
BAD_CACHE_POINTERS = [(dict(k_codes=0), NULL), (dict(v_codes=0), NULL), (dict(k_scales=0), NULL), (dict(v_scales=0), NULL),
                      (dict(k_codes=P + 8), ALIGN), (dict(v_scales=P + 1), ALIGN)]


def test_sizes():
    assert G.glowq_kv_cache_bytes(cache(k_codes=0, v_codes=0, k_scales=0, v_scales=0)) == (10 * 4 * 32 * 128, 40)
    small, large = (G.glowq_kv_attention_workspace_bytes(cache(), query(max_fresh=f)) for f in (1, 12))
    assert 0 < small and 0 < large


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_bad_caches(kw, want):
    c = cache(**kw)
    assert status(lambda: G.glowq_kv_cache_bytes(c)) == want
    assert status(lambda: G.glowq_kv_attention_workspace_bytes(c, query())) == want
    assert status(lambda: G.glowq_kv_append(c, P, 1024, P, 1024, G.GLOWQ_F16, P, 3)) == want
    assert status(lambda: G.glowq_kv_gather(c, P, 3, P, 1024, P, 1024, G.GLOWQ_F16)) == want


@pytest.mark.parametrize("kw,want", BAD_CACHE_POINTERS)
def test_bad_cache_pointers(kw, want):
    c = cache(**kw)
    assert status(lambda: G.glowq_kv_attention(c, query(), P, 1 << 30)) == want
    assert status(lambda: G.glowq_kv_append(c, P, 1024, P, 1024, G.GLOWQ_F16, P, 3)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=0), NULL), (dict(out=0), NULL), (dict(table=0), NULL), (dict(lengths=0), NULL), (dict(starts=0), NULL),
    (dict(q=P + 8), ALIGN), (dict(out=P + 2), ALIGN), (dict(table=P + 2), ALIGN),
    (dict(T=0), SHAPE), (dict(n_requests=0), SHAPE), (dict(table_width=0), SHAPE), (dict(heads=0), SHAPE), (dict(heads=6), SHAPE),
    (dict(T=1 << 20, heads=4096, ldq=1 << 20, ldo=1 << 20), SHAPE),
    (dict(ldq=1016), SHAPE), (dict(ldo=1000), SHAPE), (dict(max_fresh=0), SHAPE), (dict(max_fresh=13), SHAPE), (dict(max_length=0), SHAPE),
    (dict(window=-1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(ldq=1028), UNSUPPORTED), (dict(ldo=1036), UNSUPPORTED), (dict(act_dtype=G.GLOWQ_F32), DTYPE)])
def test_bad_queries(kw, want):
    assert status(lambda: G.glowq_kv_attention(cache(), query(**kw), P, 1 << 30)) == want


def test_workspace():
    need = G.glowq_kv_attention_workspace_bytes(cache(), query())
    assert status(lambda: G.glowq_kv_attention(cache(), query(), 0, need)) == WS
    assert status(lambda: G.glowq_kv_attention(cache(), query(), P, need - 1)) == WS
    assert status(lambda: G.glowq_kv_attention(cache(), query(), P + 128, need)) == ALIGN


@pytest.mark.parametrize("kw,want", [(dict(k=0), NULL), (dict(v=0), NULL), (dict(slots=0), NULL), (dict(k=P + 4), ALIGN),
                                     (dict(slots=P + 1), ALIGN), (dict(T=0), SHAPE), (dict(ldk=504), SHAPE), (dict(ldv=516), UNSUPPORTED),
                                     (dict(dtype=7), DTYPE)])
def test_bad_rows(kw, want):
    f = dict(k=P, v=P, slots=P, T=3, ldk=512, ldv=512, dtype=G.GLOWQ_F16)
    f.update(kw)
    assert status(lambda: G.glowq_kv_append(cache(), f["k"], f["ldk"], f["v"], f["ldv"], f["dtype"], f["slots"], f["T"])) == want
    assert status(lambda: G.glowq_kv_gather(cache(), f["slots"], f["T"], f["k"], f["ldk"], f["v"], f["ldv"], f["dtype"])) == want


def test_rows_in_32_bits_are_read_back_but_not_taken():
    assert status(lambda: G.glowq_kv_append(cache(), P, 512, P, 512, G.GLOWQ_F32, P, 3)) == DTYPE


@pytest.mark.parametrize("kw,want", [(dict([(n, 0)]), NULL) for n in ("cached", "fresh", "free_blocks", "table", "lengths", "starts",
                                                                     "slots", "positions", "taken")] +
                         [(dict(table=P + 2), ALIGN), (dict(n_requests=0), SHAPE), (dict(n_free=-1), SHAPE), (dict(table_width=0), SHAPE),
                          (dict(max_tokens=0), SHAPE), (dict(block_tokens=0), SHAPE), (dict(block_tokens=20), UNSUPPORTED)])
def test_bad_steps(kw, want):
    assert status(lambda: G.glowq_kv_plan(step(**kw))) == want


def test_descriptors_take_every_field_by_name():
    for make in (G.make_kv_step, G.make_kv_attention):
        with pytest.raises(TypeError):
            make(table=P)
