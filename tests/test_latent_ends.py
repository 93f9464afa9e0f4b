"""Latents at bfloat16's upper end: what the cache holds of finite numbers is finite, in the oracle, read back and in attention.  (Values are
E4M3 codes times 2^e; the largest that bfloat16 holds is 240 * 2^120, the next code would be 2^128.)"""
import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from oracle import kv_oracle as K
from oracle import latent_oracle as L
from gpu_util import stream
from kv_util import act_round, i32
from latent_util import Absorbed, DeviceLatents, Rows, random_latents

MOST = 240 * 2.0 ** 120
BITS = [0x7f5f, 0x7f60, 0x7f61, 0x7f6f, 0x7f70, 0x7f71, 0x7f77, 0x7f78, 0x7f79, 0x7f7e, 0x7f7f]      # up to bfloat16's largest
# Of each: its exponent, and the value that is held: codes of 2^119 have steps of 32 there, of 2^120 of 16
HELD = [(119, 448 * 2.0 ** 119), (119, 448 * 2.0 ** 119)] + [(120, 224 * 2.0 ** 120)] + [(120, MOST)] * 8


def tokens(rng, latent):
    """(latents, one with each of the numbers, alone, negative or everywhere)"""
    top = np.array(BITS, np.uint32).__lshift__(16).view(np.float32).astype(np.float64)
    c = np.zeros((3 * len(BITS), latent))
    for i, v in enumerate(top):
        c[3 * i:3 * i + 2] = rng.uniform(-1, 1, (2, latent)) * v
        c[3 * i, 5], c[3 * i + 1, latent - 3], c[3 * i + 2] = v, -v, v
    return act_round(c, "bf16")


def test_the_oracle_holds_numbers():
    c = tokens(np.random.default_rng(1), 256)
    cache = L.LatentCache(3, 16, 256, 32, "bf16")
    cache.append(c, np.zeros((len(c), 32)), np.arange(len(c)))
    held = cache.latents(np.arange(len(c)))
    assert np.isfinite(act_round(held, "bf16")).all() and np.array_equal(act_round(held, "bf16"), held)
    for i, (e, v) in enumerate(HELD):
        assert (cache.exps[3 * i:3 * i + 3] == e).all() and held[3 * i, 5] == v and held[3 * i + 1, 253] == -v and (held[3 * i + 2] == v).all()
    # what is no number stays none
    c[0, 7], c[1, 8] = np.inf, np.nan
    cache.append(c[:2], np.zeros((2, 32)), [0, 1])
    assert np.isnan(K.VALUES[cache.codes[0, 7]]) and np.isnan(K.VALUES[cache.codes[1, 8]]) and np.isfinite(cache.latents([0])[0, :7]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("latent", [256, 512])
def test_into_the_cache_and_back(latent):
    rng = np.random.default_rng(2)
    c = tokens(rng, latent)
    T = len(c)
    c[1, 7], c[2, 8] = np.inf, np.nan
    d = DeviceLatents(random_latents(rng, 3, 16, latent, 32, "bf16"))
    dc, dr, slots = Rows(c[:, None], "bf16"), Rows(np.zeros((T, 1, 32)), "bf16"), i32(np.arange(T))
    G.glowq_latent_append(d.desc, None, None, dc.buf.data_ptr(), dc.ld, dr.buf.data_ptr(), dr.ld, slots.data_ptr(), 0, T, stream())
    back, br = Rows(np.zeros((T, 1, latent)), "bf16", filled=False), Rows(np.zeros((T, 1, 32)), "bf16", filled=False)
    G.glowq_latent_gather(d.desc, slots.data_ptr(), T, back.buf.data_ptr(), back.ld, br.buf.data_ptr(), br.ld, stream())
    got = back.numbers()[:, 0]
    assert np.array_equal(np.isfinite(got), np.isfinite(c))
    d.o.append(c, np.zeros((T, 32)), np.arange(T))
    assert np.array_equal(got, d.o.latents(np.arange(T)), equal_nan=True)
    assert np.array_equal(d.scales.cpu().numpy()[:T], (d.o.exps[:T] + 127).astype(np.uint8))
    for i, (e, v) in enumerate(HELD):
        assert got[3 * i, 5] == v and got[3 * i + 1, latent - 3] == -v


@pytest.mark.gpu
@pytest.mark.parametrize("heads,latent", [(5, 512), (40, 256)])
def test_attention_over_them(heads, latent):
    rng = np.random.default_rng(3)
    b = Absorbed(rng, [(700, 3), (40, 1)], heads, latent, 32, 16, "bf16")
    n = b.cache.n_blocks * 16
    c = np.tile(tokens(rng, latent), (n // (3 * len(BITS)) + 1, 1))[rng.permutation(n)]
    parts = act_round(rng.standard_normal((n, 32)), "bf16")
    b.cache.append(c, parts, np.arange(n))
    # scores of about one, from numbers that are not subnormal
    b.q[..., :latent] *= 2.0 ** -122
    b.q[np.abs(b.q) < 2.0 ** -126] = 0
    b.scale = 1.0 / 512
    b.device()
    codes, scales = b.dc.codes.clone(), b.dc.scales.clone()
    dc, dr, slots = Rows(c[:, None], "bf16"), Rows(parts[:, None], "bf16"), i32(np.sort(b.used))
    at = slots.long()
    dc.buf[:len(at)], dr.buf[:len(at)] = dc.buf[at].clone(), dr.buf[at].clone()
    G.glowq_latent_append(b.dc.desc, None, None, dc.buf.data_ptr(), dc.ld, dr.buf.data_ptr(), dr.ld, slots.data_ptr(), 0, len(at), stream())
    torch.cuda.synchronize()
    assert torch.equal(b.dc.codes, codes) and torch.equal(b.dc.scales, scales)          # as the oracle has them
    out = b.run().check()
    assert np.isfinite(out).all() and np.abs(out).max() > 2.0 ** 124
