"""Rotary rows whose heads lie 2 GiB and more apart: every entry point that takes such rows, as inputs, as outputs and in place."""
import numpy as np
import pytest
import torch

import paper_2603_25385_amd as G
from gpu_util import ACT_CODE, TORCH_ACT, stream
from kv_util import DeviceCache, i32, random_cache
from latent_util import DeviceLatents, Rope, random_latents
from test_gpu_rope import check_rotated, numbers

pytestmark = pytest.mark.gpu
T, HEADS = 2, 2


def spread(act, lh, d):
    """(rows of two heads lh numbers apart, what holds them)"""
    mem = torch.empty((T - 1) * (lh + d) + lh + d, dtype=TORCH_ACT[act], device="cuda")
    return mem.as_strided((T, HEADS, d), (lh + d, lh, 1)), mem


def rows(x, y):
    return G.make_rope_rows(x=x.data_ptr(), y=y.data_ptr(), heads=HEADS, ldx=x.stride(0), lhx=x.stride(1), ldy=y.stride(0), lhy=y.stride(1))


@pytest.mark.parametrize("act,lh,entry", [("f16", 1 << 30, "rotate"), ("bf16", (1 << 30) + 64, "kv"), ("f16", 1 << 30, "latent"), ("f32", 1 << 29, "rotate"),
                                          ("f32", (1 << 30) - 8, "rotate")])
def test_heads_far_apart(act, lh, entry):
    rng, d = np.random.default_rng(lh % 1000), 64
    rope, positions, slots = Rope(64, "pairs"), np.array([5, 70000]), i32([3, 40])
    at, x = i32(positions), numbers(rng, T, HEADS, d, act)
    far, mem = spread(act, lh, d)
    near = torch.empty(T, HEADS, d, dtype=TORCH_ACT[act], device="cuda")
    kv, lat = DeviceCache(random_cache(rng, 4, 16, 2, d)), DeviceLatents(random_latents(rng, 4, 16, 256, d, "f16" if act == "f32" else act))
    new = torch.randn(T, 256 + d, device="cuda").to(near.dtype)

    def call(q):
        if entry == "rotate":
            G.glowq_rotate(rope.desc, [q], d, ACT_CODE[act], at.data_ptr(), T, stream())
        elif entry == "kv":
            G.glowq_kv_append_rotated(kv.desc, rope.desc, q, new.data_ptr(), 256 + d, new.data_ptr(), 256 + d, ACT_CODE[act], slots.data_ptr(), at.data_ptr(), T, stream())
        else:
            G.glowq_latent_append(lat.desc, rope.desc, q, new.data_ptr(), 256 + d, new.data_ptr() + 512, 256 + d, slots.data_ptr(), at.data_ptr(), T, stream())
        torch.cuda.synchronize()

    given = torch.from_numpy(x).to(near.dtype).cuda()
    far.copy_(given)
    call(rows(far, near))                                          # from far apart
    check_rotated(rope, x, near.double().cpu().numpy(), positions, act)
    assert torch.equal(far, given)
    want = near.clone()
    far.fill_(float("nan"))
    near.copy_(given)
    call(rows(near, far))                                          # to far apart
    assert torch.equal(far, want) and torch.equal(near, given)
    far.copy_(given)
    call(rows(far, far))                                           # in place
    assert torch.equal(far, want) and mem.numel() > 1 << 29
