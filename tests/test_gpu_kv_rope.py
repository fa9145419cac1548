"""mq_qk_norm_rope_scaled (rotary embedding of part of a head, scaled frequencies) against the float64 definition.

Tolerance: that of mq_qk_norm_rope's tests, half a bf16 step of the result and fewer than 32 float32 roundings relative to the magnitudes a
result is made of (the factor amp is one of them); channels that pass without a norm keep their bits.
"""
import numpy as np
import pytest
import torch

from oracle import kv_oracle as O
from paper_2502_00425_b200 import binding as B

from kv_util import DEV

pytestmark = pytest.mark.gpu


def _bf16(rng, *shape):
    return torch.from_numpy((rng.standard_normal(shape) * 3).astype(np.float32)).to(torch.bfloat16)


def _call(q, k, v, pos, hq, hkv, rope, dim, gains=(None, None), int8=False, page=16):
    T = q.shape[0]
    n_pages = T // page + 2
    pool = [torch.full((n_pages, hkv, page, dim), 99, dtype=torch.int8 if int8 else torch.bfloat16, device=DEV) for _ in range(2)]
    scales = [torch.linspace(0.02, 0.05, hkv, device=DEV) for _ in range(2)] if int8 else [None, None]
    cache = B.KVCache(*pool, *scales)
    slots = torch.from_numpy(np.random.default_rng(T).permutation(n_pages * page)[:T].astype(np.int64))
    q_out, k_out = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    B.mq_qk_norm_rope_scaled(q.to(DEV), k.to(DEV), torch.from_numpy(pos).to(DEV), hq, hkv, q_out, rope, k_out=k_out,
                             gain_q=None if gains[0] is None else torch.from_numpy(gains[0]).to(DEV),
                             gain_k=None if gains[1] is None else torch.from_numpy(gains[1]).to(DEV), v=v.to(DEV), cache=cache, slots=slots.to(DEV))
    torch.cuda.synchronize()
    rows = [p.permute(0, 2, 1, 3).reshape(-1, hkv, dim).cpu()[slots] for p in pool]
    return q_out.cpu(), k_out.cpu(), rows, scales


@pytest.mark.parametrize("T,hq,hkv,dim,rot,half,norm,int8,far,factor,original", [
    (1, 28, 4, 128, 128, True, False, False, 70000, 4.0, 32768),
    (5, 4, 2, 64, 16, True, True, False, 0, 1.0, 0),
    (33, 32, 8, 128, 64, True, True, False, 1 << 20, 8.0, 0),
    (33, 3, 3, 64, 40, False, False, True, 30000, 2.0, 4096),     # an odd share of the head
    (7, 28, 4, 128, 8, False, True, True, 1 << 30, 8.0, 4096),    # one pair block, far out
    (9, 8, 2, 128, 0, True, True, False, 5, 1.0, 0),              # nothing rotates
    (1300, 12, 4, 64, 24, True, True, True, 100000, 4.0, 8192),   # many rows: the variant with several loads in flight
    (2300, 5, 1, 128, 104, True, False, False, 1000, 1.0, 0),
    (2300, 5, 1, 128, 104, False, True, False, 1000, 3.0, 0),
])
def test_scaled_rotary(T, hq, hkv, dim, rot, half, norm, int8, far, factor, original):
    rng = np.random.default_rng(T + dim + rot)
    q, k, v = _bf16(rng, T, hq * dim), _bf16(rng, T, hkv * dim), _bf16(rng, T, hkv * dim)
    pos = (rng.permutation(T) + far).astype(np.int32)
    gains = tuple((1 + 0.2 * rng.standard_normal(dim)).astype(np.float32) if norm else None for _ in range(2))
    amp = 0.1 * np.log(factor) + 1.0
    rope = B.Rope(rot, half=half, factor=factor, original=original, amp=amp)
    q_out, k_out, (kc, vc), scales = _call(q, k, v, pos, hq, hkv, rope, dim, gains, int8)
    theta = O.rope_theta(rot, 10000.0, factor, original)
    for x, got, h, gain in ((q, q_out, hq, gains[0]), (k, k_out, hkv, gains[1])):
        y, mag = O.norm_rope_scaled(x.double().numpy().reshape(T, h, dim), gain, 1e-6, pos, theta, half, amp)
        g = got.double().numpy().reshape(T, h, dim)
        assert np.all(np.abs(g - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -19 * mag + 1e-38)
        if not norm:
            assert torch.equal(got.view(T, h, dim)[..., rot:], x.view(T, h, dim)[..., rot:])
    if not int8:
        assert torch.equal(kc, k_out.view(T, hkv, dim)) and torch.equal(vc, v.view(T, hkv, dim))
    else:
        s = scales[0].double().cpu().numpy()[:, None]
        assert np.all(np.abs(kc.double().numpy() - np.clip(y / s, -128, 127)) <= 0.5 + 2.0 ** -19 * mag / s + 2.0 ** -22 * np.abs(y / s))
        want = np.clip(v.double().numpy().reshape(T, hkv, dim) / s, -128, 127)
        assert np.all(np.abs(vc.double().numpy() - want) <= 0.5 + 2.0 ** -21 * np.abs(want))


@pytest.mark.parametrize("half", [False, True])
def test_the_whole_head_unscaled_is_the_plain_call(half):
    """The same kernel and, to a rounding of a double, the same frequencies."""
    rng = np.random.default_rng(3)
    T, hq, hkv, dim = 40, 6, 2, 128
    q, k, v = _bf16(rng, T, hq * dim), _bf16(rng, T, hkv * dim), _bf16(rng, T, hkv * dim)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    q_out, k_out, _, _ = _call(q, k, v, pos, hq, hkv, B.Rope(dim, half=half), dim)
    q2, k2 = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    B.mq_qk_norm_rope(q.to(DEV), k.to(DEV), torch.from_numpy(pos).to(DEV), hq, hkv, q2, k_out=k2, half=half)
    for x, got, want in ((q, q_out, q2.cpu()), (k, k_out, k2.cpu())):
        # both are within half a bf16 step (and the arithmetic in front of it) of the same number
        pairs = x.double().view(T, -1, dim)
        mag = (pairs.abs() + (pairs.roll(dim // 2, -1) if half else pairs.view(T, -1, dim // 2, 2).flip(-1).reshape(pairs.shape)).abs()).view(T, -1)
        assert bool(((got.double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs() + 2.0 ** -18 * mag).all())


@pytest.mark.parametrize("half", [False, True])
def test_infinities_and_nans_of_passing_channels_stay_where_they_are(half):
    rng = np.random.default_rng(4)
    T, hq, hkv, dim, rot = 6, 4, 2, 64, 24
    q, k, v = _bf16(rng, T, hq * dim), _bf16(rng, T, hkv * dim), _bf16(rng, T, hkv * dim)
    q.view(T, hq, dim)[:, :, rot] = float("inf")
    q.view(T, hq, dim)[:, :, dim - 1] = float("nan")
    q_out, _, _, _ = _call(q, k, v, np.arange(T, dtype=np.int32), hq, hkv, B.Rope(rot, half=half), dim)
    a, b = q_out.view(T, hq, dim), q.view(T, hq, dim)
    assert bool(torch.isfinite(a[..., :rot]).all()) and torch.equal(a[..., rot:dim - 1], b[..., rot:dim - 1]) and bool(a[..., dim - 1].isnan().all())


def test_captured_with_the_frequencies_of_its_time():
    rng = np.random.default_rng(6)
    T, hq, hkv, dim = 12, 4, 2, 128
    q, k = _bf16(rng, T, hq * dim).to(DEV), _bf16(rng, T, hkv * dim).to(DEV)
    pos = torch.zeros(T, dtype=torch.int32, device=DEV)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    rope = B.Rope(64, factor=2.0)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.mq_qk_norm_rope_scaled(q, k, pos, hq, hkv, q_out, rope, k_out=k_out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mq_qk_norm_rope_scaled(q, k, pos, hq, hkv, q_out, rope, k_out=k_out)
    del rope                                     # (the call read its array; a replay does not)
    pos.copy_(torch.arange(T, device=DEV) * 1000)
    graph.replay()
    torch.cuda.synchronize()
    y, mag = O.norm_rope_scaled(q.double().cpu().numpy().reshape(T, hq, dim), None, 0, pos.cpu().numpy(), O.rope_theta(64, 10000.0, 2.0), False, 1.0)
    got = q_out.double().cpu().numpy().reshape(T, hq, dim)
    assert np.all(np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -19 * mag)
