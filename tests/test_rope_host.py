"""Refusals of rotary positions and of the latent operators: documented status codes, before any device is touched."""
import pytest

import paper_2603_25385_amd as G

P = 0x1000
NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED, WS = (G.GLOWQ_ERR_NULL, G.GLOWQ_ERR_SHAPE, G.GLOWQ_ERR_ALIGN, G.GLOWQ_ERR_DTYPE,
                                              G.GLOWQ_ERR_UNSUPPORTED, G.GLOWQ_ERR_WORKSPACE)


def status(call):
    with pytest.raises(G.GlowqError) as e:
        call()
    return e.value.status


def changed(make, base, kw):
    return make(**{**base, **kw})


SPEC = dict(rotary_dim=64, scaling=G.GLOWQ_ROPE_BANDS, base=10000.0, factor=4.0, low=1.0, high=4.0, trained_length=4096)
ROPE = dict(turns=P, rotary_dim=64, layout=G.GLOWQ_ROPE_HALVES, magnitude=1.0)
ROWS = dict(x=P, y=P + 64, heads=4, ldx=512, lhx=128, ldy=512, lhy=128)
KV = dict(k_codes=P, v_codes=P, k_scales=P, v_scales=P, n_blocks=10, block_tokens=32, kv_heads=4, head_dim=128)
LATENT = dict(codes=P, scales=P, ropes=P, n_blocks=10, block_tokens=32, latent_dim=512, rope_dim=64, act_dtype=G.GLOWQ_BF16)
QUERY = dict(q=P, out=P, table=P, lengths=P, starts=P, ldq=8 * 576, ldo=8 * 512, table_width=8, n_requests=3, T=12, heads=8, max_fresh=4,
             max_length=200, scale=0.1)
EXPANDED = dict(q=P, k=P, k_rope=P, v=P, out=P, starts=P, key_starts=P, lengths=P, ldq=8 * 192, lhq=192, ldk=8 * 256, lhk=256, ldr=64,
                ldv=8 * 256, lhv=256, ldo=8 * 128, n_requests=3, T=12, keys=600, heads=8, nope_dim=128, rope_dim=64, v_dim=128,
                act_dtype=G.GLOWQ_F16, max_fresh=4, max_length=600, scale=0.1)


@pytest.mark.parametrize("kw,want", [
    (dict(rotary_dim=0), SHAPE), (dict(rotary_dim=15), SHAPE), (dict(rotary_dim=8192), SHAPE), (dict(rotary_dim=24), UNSUPPORTED),
    (dict(base=1.0), SHAPE), (dict(base=float("nan")), SHAPE), (dict(base=float("inf")), SHAPE), (dict(scaling=-1), SHAPE), (dict(scaling=5), SHAPE),
    (dict(factor=0.5), SHAPE), (dict(factor=float("nan")), SHAPE), (dict(factor=float("inf")), SHAPE), (dict(low=0.0), SHAPE),
    (dict(high=1.0), SHAPE), (dict(high=float("inf")), SHAPE), (dict(trained_length=0), SHAPE),
    (dict(scaling=G.GLOWQ_ROPE_RAMP, low=float("nan")), SHAPE), (dict(scaling=G.GLOWQ_ROPE_REBASED, factor=0.0), SHAPE)])
def test_bad_specs(kw, want):
    assert status(lambda: G.glowq_rope_turns(changed(G.make_rope_spec, SPEC, kw))) == want


def test_specs_that_ignore_fields():
    turns, magnitude = G.glowq_rope_turns(changed(G.make_rope_spec, SPEC, dict(scaling=G.GLOWQ_ROPE_PLAIN, factor=0.0, low=-1.0, trained_length=-1)))
    assert len(turns) == 32 and magnitude == 1.0 and turns[0] > turns[-1] > 0


BAD_ROPES = [(dict(turns=0), NULL), (dict(turns=P + 4), ALIGN), (dict(rotary_dim=0), SHAPE), (dict(rotary_dim=17), SHAPE), (dict(rotary_dim=272), SHAPE),
             (dict(rotary_dim=24), UNSUPPORTED), (dict(layout=2), SHAPE), (dict(layout=-1), SHAPE), (dict(magnitude=float("nan")), SHAPE),
             (dict(magnitude=float("inf")), SHAPE)]
BAD_ROWS = [(dict(x=0), NULL), (dict(y=0), NULL), (dict(x=P + 8), ALIGN), (dict(y=P + 2), ALIGN), (dict(heads=0), SHAPE), (dict(heads=4097), SHAPE),
            (dict(lhx=120), SHAPE), (dict(lhy=64), SHAPE), (dict(ldx=504), SHAPE), (dict(ldy=384), SHAPE), (dict(ldx=516), UNSUPPORTED),
            (dict(lhx=132, ldx=1024), UNSUPPORTED), (dict(y=P, ldy=1024), SHAPE), (dict(y=P, lhy=136, ldy=1024), SHAPE)]


@pytest.mark.parametrize("kw,want", BAD_ROPES)
def test_bad_ropes(kw, want):
    rope, rows = changed(G.make_rope, ROPE, kw), G.make_rope_rows(**ROWS)
    assert status(lambda: G.glowq_rotate(rope, [rows], 128, G.GLOWQ_F16, P, 3)) == want
    assert status(lambda: G.glowq_kv_append_rotated(G.make_kv_cache(**KV), rope, None, P, 512, P, 512, G.GLOWQ_F16, P, P, 3)) == want
    assert status(lambda: G.glowq_latent_append(G.make_latent_cache(**LATENT), rope, None, P, 512, P, 64, P, P, 3)) == want


@pytest.mark.parametrize("kw,want", BAD_ROWS)
def test_bad_rows(kw, want):
    rope, rows = G.make_rope(**ROPE), changed(G.make_rope_rows, ROWS, kw)
    assert status(lambda: G.glowq_rotate(rope, [G.make_rope_rows(**ROWS), rows], 128, G.GLOWQ_F32, P, 3)) == want
    assert status(lambda: G.glowq_kv_append_rotated(G.make_kv_cache(**KV), rope, rows, P, 512, P, 512, G.GLOWQ_F16, P, P, 3)) == want


def test_bad_rotations():
    rope, rows = G.make_rope(**ROPE), G.make_rope_rows(**ROWS)
    call = lambda rope=rope, rows=[rows], dim=128, dtype=G.GLOWQ_F16, positions=P, T=3: G.glowq_rotate(rope, rows, dim, dtype, positions, T)
    for kw, want in ((dict(rope=None), NULL), (dict(rows=[]), SHAPE), (dict(rows=[rows] * 5), SHAPE), (dict(dim=0), SHAPE), (dict(dim=8192), SHAPE),
                     (dict(dim=72), UNSUPPORTED), (dict(dtype=3), DTYPE), (dict(positions=0), NULL), (dict(positions=P + 2), ALIGN), (dict(T=0), SHAPE),
                     (dict(T=(1 << 20) + 1), SHAPE)):
        assert status(lambda: call(**kw)) == want, kw
    # more threads than a launch counts
    wide = G.make_rope_rows(x=P, y=P, heads=4096, ldx=4096 * 4096, lhx=4096, ldy=4096 * 4096, lhy=4096)
    assert status(lambda: call(rows=[wide] * 4, dim=4096, T=1 << 20)) == SHAPE


def test_bad_rotated_appends():
    rope = G.make_rope(**ROPE)
    base = dict(cache=G.make_kv_cache(**KV), rope=rope, q=None, k=P, ldk=512, v=P, ldv=512, act_dtype=G.GLOWQ_F16, slots=P, positions=P, T=3)
    for kw, want in ((dict(rope=None), NULL), (dict(k=0), NULL), (dict(v=0), NULL), (dict(slots=0), NULL), (dict(positions=0), NULL), (dict(k=P + 4), ALIGN),
                     (dict(positions=P + 1), ALIGN), (dict(T=0), SHAPE), (dict(ldk=504), SHAPE), (dict(ldv=516), UNSUPPORTED),
                     (dict(act_dtype=G.GLOWQ_F32), DTYPE), (dict(cache=changed(G.make_kv_cache, KV, dict(head_dim=96))), UNSUPPORTED)):
        assert status(lambda: G.glowq_kv_append_rotated(**{**base, **kw})) == want, kw


BAD_LATENTS = [(dict(n_blocks=0), SHAPE), (dict(latent_dim=0), SHAPE), (dict(rope_dim=0), SHAPE), (dict(block_tokens=0), SHAPE), (dict(block_tokens=48), UNSUPPORTED),
               (dict(latent_dim=384), UNSUPPORTED), (dict(rope_dim=128), UNSUPPORTED), (dict(n_blocks=1 << 27), SHAPE), (dict(act_dtype=G.GLOWQ_F32), DTYPE)]


@pytest.mark.parametrize("kw,want", BAD_LATENTS)
def test_bad_latent_caches(kw, want):
    c = changed(G.make_latent_cache, LATENT, kw)
    assert status(lambda: G.glowq_latent_cache_bytes(c)) == want
    assert status(lambda: G.glowq_latent_attention_workspace_bytes(c, G.make_latent_attention(**QUERY))) == want
    assert status(lambda: G.glowq_latent_append(c, None, None, P, 512, P, 128, P, 0, 3)) == want
    assert status(lambda: G.glowq_latent_gather(c, P, 3, P, 512, P, 128)) == want


@pytest.mark.parametrize("kw,want", [(dict(codes=0), NULL), (dict(scales=0), NULL), (dict(ropes=0), NULL), (dict(codes=P + 8), ALIGN), (dict(scales=P + 4), ALIGN),
                                     (dict(ropes=P + 8), ALIGN)])
def test_bad_latent_cache_pointers(kw, want):
    c = changed(G.make_latent_cache, LATENT, kw)
    assert status(lambda: G.glowq_latent_attention(c, G.make_latent_attention(**QUERY), P, 1 << 40)) == want
    assert status(lambda: G.glowq_latent_append(c, None, None, P, 512, P, 64, P, 0, 3)) == want


def test_latent_sizes():
    assert G.glowq_latent_cache_bytes(changed(G.make_latent_cache, LATENT, dict(codes=0, scales=0, ropes=0))) == (320 * 512, 320, 320 * 128)


def test_bad_latent_rows():
    base = dict(cache=G.make_latent_cache(**LATENT), rope=G.make_rope(**ROPE), q=None, c=P, ldc=576, r=P, ldr=576, slots=P, positions=P, T=3)
    rows = G.make_rope_rows(x=P, y=P, heads=2, ldx=384, lhx=192, ldy=384, lhy=192)
    for kw, want in ((dict(c=0), NULL), (dict(r=0), NULL), (dict(slots=0), NULL), (dict(positions=0), NULL), (dict(c=P + 8), ALIGN), (dict(r=P + 2), ALIGN),
                     (dict(slots=P + 1), ALIGN), (dict(positions=P + 2), ALIGN), (dict(T=0), SHAPE), (dict(ldc=504), SHAPE), (dict(ldr=56), SHAPE),
                     (dict(ldc=580), UNSUPPORTED), (dict(rope=None, q=rows), NULL), (dict(rope=changed(G.make_rope, ROPE, dict(rotary_dim=80))), SHAPE),
                     (dict(q=changed(G.make_rope_rows, ROWS, dict(lhx=48))), SHAPE)):
        assert status(lambda: G.glowq_latent_append(**{**base, **kw})) == want, kw
    for kw, want in ((dict(c=0), NULL), (dict(r=0), NULL), (dict(slots=0), NULL), (dict(c=P + 4), ALIGN), (dict(T=0), SHAPE), (dict(ldc=504), SHAPE),
                     (dict(ldr=68), UNSUPPORTED)):
        g = {k: base[k] for k in ("cache", "slots", "T", "c", "ldc", "r", "ldr")}
        assert status(lambda: G.glowq_latent_gather(**{**g, **kw})) == want, kw


def test_bad_head_maps():
    base = dict(x=P, ldx=384, lhx=192, w=P, y=P, ldy=1152, lhy=576, heads=2, d_in=128, d_out=512, act_dtype=G.GLOWQ_F16, T=3)
    for kw, want in ((dict(x=0), NULL), (dict(w=0), NULL), (dict(y=0), NULL), (dict(w=P + 8), ALIGN), (dict(T=0), SHAPE), (dict(T=(1 << 20) + 1), SHAPE),
                     (dict(heads=0), SHAPE), (dict(d_in=0), SHAPE), (dict(d_out=0), SHAPE), (dict(lhx=120), SHAPE), (dict(lhy=504), SHAPE), (dict(ldx=312), SHAPE),
                     (dict(ldy=1080), SHAPE), (dict(d_in=112), UNSUPPORTED), (dict(d_out=504), UNSUPPORTED), (dict(ldx=388), UNSUPPORTED),
                     (dict(act_dtype=G.GLOWQ_F32), DTYPE)):
        assert status(lambda: G.glowq_head_maps(**{**base, **kw})) == want, kw


@pytest.mark.parametrize("kw,want", [
    (dict(q=0), NULL), (dict(out=0), NULL), (dict(table=0), NULL), (dict(lengths=0), NULL), (dict(starts=0), NULL), (dict(q=P + 8), ALIGN),
    (dict(table=P + 2), ALIGN), (dict(T=0), SHAPE), (dict(n_requests=0), SHAPE), (dict(table_width=0), SHAPE), (dict(heads=0), SHAPE), (dict(heads=1025), SHAPE),
    (dict(ldq=8 * 576 - 8), SHAPE), (dict(ldo=8 * 512 - 8), SHAPE), (dict(max_fresh=0), SHAPE), (dict(max_fresh=13), SHAPE), (dict(max_length=0), SHAPE),
    (dict(scale=0.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(ldq=8 * 576 + 4), UNSUPPORTED)])
def test_bad_latent_queries(kw, want):
    assert status(lambda: G.glowq_latent_attention(G.make_latent_cache(**LATENT), changed(G.make_latent_attention, QUERY, kw), P, 1 << 40)) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=0), NULL), (dict(k=0), NULL), (dict(k_rope=0), NULL), (dict(v=0), NULL), (dict(out=0), NULL), (dict(starts=0), NULL), (dict(key_starts=0), NULL),
    (dict(lengths=0), NULL), (dict(k=P + 8), ALIGN), (dict(key_starts=P + 2), ALIGN), (dict(T=0), SHAPE), (dict(n_requests=0), SHAPE), (dict(keys=0), SHAPE),
    (dict(heads=0), SHAPE), (dict(nope_dim=0), SHAPE), (dict(nope_dim=96), UNSUPPORTED), (dict(v_dim=64), UNSUPPORTED), (dict(rope_dim=16), UNSUPPORTED),
    (dict(lhq=184), SHAPE), (dict(lhk=120), SHAPE), (dict(lhv=120), SHAPE), (dict(ldq=1528), SHAPE), (dict(ldk=1912), SHAPE), (dict(ldv=1912), SHAPE),
    (dict(ldr=56), SHAPE), (dict(ldo=1016), SHAPE), (dict(ldk=(1 << 24) + 8), SHAPE), (dict(ldq=1540), UNSUPPORTED), (dict(lhk=260, ldk=2080), UNSUPPORTED),
    (dict(act_dtype=G.GLOWQ_F32), DTYPE), (dict(max_fresh=13), SHAPE), (dict(max_length=0), SHAPE), (dict(scale=-1.0), SHAPE)])
def test_bad_expanded_queries(kw, want):
    assert status(lambda: G.glowq_expanded_attention(changed(G.make_expanded_attention, EXPANDED, kw), P, 1 << 40)) == want


def test_workspaces():
    c, q, e = G.make_latent_cache(**LATENT), G.make_latent_attention(**QUERY), G.make_expanded_attention(**EXPANDED)
    for need, call in ((G.glowq_latent_attention_workspace_bytes(c, q), lambda p, n: G.glowq_latent_attention(c, q, p, n)),
                       (G.glowq_expanded_attention_workspace_bytes(e), lambda p, n: G.glowq_expanded_attention(e, p, n))):
        assert need > 0 and status(lambda: call(0, need)) == WS and status(lambda: call(P, need - 1)) == WS and status(lambda: call(P + 128, need)) == ALIGN


def test_descriptors_take_every_field_by_name():
    for make in (G.make_rope_spec, G.make_rope, G.make_rope_rows, G.make_latent_cache, G.make_latent_attention, G.make_expanded_attention):
        with pytest.raises(TypeError):
            make(heads=P)
