"""GPU: ff_rotary against the float64 oracle.  A result is two products and a sum in float32, with sine and cosine two steps off at
most and the angle reduced in float64, and is rounded to the type once."""
import numpy as np
import pytest
import torch

import oracle
import paper_2301_08739_amd as ff
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def _check(dtype, got, x, positions, freqs, half, amplitude=1.0, inverse=False):
    x = x.detach().double().cpu().numpy()
    p, f = positions.cpu().numpy().reshape(x.shape[0], -1), freqs.cpu().numpy()
    want = oracle.rotary(x, p, f, half, amplitude, inverse)
    size = oracle.rotary(np.abs(x), 0 * p, f, half, abs(amplitude))
    turned = 2 * f.size
    pair = size.copy()                                  # |a| + |b| of every pair
    for c in range(f.shape[0]):
        seg = size[..., 2 * f.shape[1] * c:2 * f.shape[1] * (c + 1)]
        both = seg[..., :f.shape[1]] + seg[..., f.shape[1]:] if half else seg[..., 0::2] + seg[..., 1::2]
        pair[..., 2 * f.shape[1] * c:2 * f.shape[1] * (c + 1)] = np.concatenate([both, both], -1) if half else np.repeat(both, 2, -1)
    # the angle: 2^-24 of a turn for its float32 fraction (half a turn at most), and float64's 2^-53 of all turns
    turns = np.abs(p[:, :, None] * f / (2 * np.pi)).max(initial=0) * 2.0 ** -52
    bound = HALF_STEP[dtype] * np.abs(want) + pair * (8 * 2.0 ** -24 + 2 * np.pi * (2.0 ** -25 + turns)) + (2.0 ** -25 if dtype == "f16" else 2.0 ** -126)
    got = got.detach().double().cpu().numpy()
    assert (got[..., turned:] == x[..., turned:]).all()
    bad = np.abs(got - want) > bound
    assert not bad[..., :turned].any(), (int(bad.sum()), np.abs(got - want).max())


def _rows(dtype, rng, n, h, d):
    return torch.from_numpy(rng.standard_normal((n, h, d))).to(TYPES[dtype]).to(DEV)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("D,axes,pairs", [(2, 1, 1), (16, 2, 4), (16, 1, 8), (16, 1, 3), (24, 3, 4), (32, 2, 8), (48, 3, 7), (64, 1, 16), (80, 1, 40),
                                          (128, 1, 64), (128, 2, 32), (130, 1, 1), (256, 1, 128), (33, 2, 8)])
def test_shapes(dtype, half, D, axes, pairs):
    rng = np.random.default_rng(D)
    for n, H, K in ((1, 1, 1), (37, 4, 2), (301, 3, 0)):
        q, k = _rows(dtype, rng, n, H, D), _rows(dtype, rng, n, K, D) if K else None
        p = torch.from_numpy(rng.integers(-400, 400, (n, axes)).astype(np.int32)).to(DEV)
        f = torch.from_numpy(rng.uniform(0, 3, (axes, pairs))).to(DEV)
        layout = ff.FF_ROTARY_HALF if half else ff.FF_ROTARY_INTERLEAVED
        q2, k2 = ff.ff_rotary(q, k, p, f, layout=layout)
        _check(dtype, q2, q, p, f, half)
        if K:
            _check(dtype, k2, k, p, f, half)
        q3, _ = ff.ff_rotary(q, None, p, f, layout=layout, amplitude=1.25, inverse=True)
        _check(dtype, q3, q, p, f, half, 1.25, True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("half", [True, False])
def test_views_in_place_and_positions_of_coordinates(dtype, half):
    rng = np.random.default_rng(5)
    n, H, K, D = 500, 4, 2, 32
    layout = ff.FF_ROTARY_HALF if half else ff.FF_ROTARY_INTERLEAVED
    coords = torch.from_numpy(rng.integers(0, 468, (n, 3)).astype(np.int32)).to(DEV)
    f = ff.ff_rotary_frequencies(8, axes=2)
    packed = _rows(dtype, rng, n, H + 2 * K, D)
    before = packed.clone()
    q, k = packed[:, :H], packed[:, H:H + K]
    a, b = ff.ff_rotary(q, k, coords[:, 1:], f, layout=layout)                 # out of place
    ff.ff_rotary(q, k, coords[:, 1:], f, layout=layout, q_out=q, k_out=k)      # in place, the same bits
    assert torch.equal(q, a) and torch.equal(k, b) and torch.equal(packed[:, H + K:], before[:, H + K:])
    _check(dtype, a, before[:, :H], coords[:, 1:], f, half)
    turned = before.transpose(0, 1).contiguous().transpose(0, 1)               # heads first
    c, _ = ff.ff_rotary(turned[:, :H], None, coords[:, 1:], f, layout=layout)
    assert torch.equal(c, a)
    odd = torch.zeros(n, H, D + 3, dtype=packed.dtype, device=DEV)[:, :, 1:1 + D].copy_(before[:, :H])
    d, _ = ff.ff_rotary(odd, None, coords.T.contiguous().T[:, 1:], f, layout=layout)
    assert torch.equal(d, a)


@pytest.mark.parametrize("dtype", TYPES)
def test_far_positions_keep_their_precision(dtype):
    rng = np.random.default_rng(6)
    p = torch.tensor([0, 1, 2 ** 20 + 1, 2 ** 30 + 7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV)
    f = ff.ff_rotary_frequencies(32, factor=8.0, original_length=8192)
    q = _rows(dtype, rng, 6, 2, 64)
    q2, _ = ff.ff_rotary(q, None, p, f)
    _check(dtype, q2, q, p, f, True)
    back, _ = ff.ff_rotary(q2, None, p, f, inverse=True)
    assert (back.double() - q.double()).abs().max() <= 8 * (2 * HALF_STEP[dtype] + 2.0 ** -20)


def test_nothing_to_turn_and_many_rows():
    f = ff.ff_rotary_frequencies(8)
    empty = torch.empty(0, 2, 16, device=DEV)
    a, b = ff.ff_rotary(empty, empty, torch.empty(0, dtype=torch.int32, device=DEV), f)
    assert a.shape == b.shape == (0, 2, 16)
    rng = np.random.default_rng(7)
    q = _rows("bf16", rng, 70001, 2, 16)
    p = torch.arange(70001, dtype=torch.int32, device=DEV)
    _check("bf16", ff.ff_rotary(q, None, p, f)[0], q, p, f, True)


def test_in_a_graph():
    rng = np.random.default_rng(8)
    q, k = _rows("f16", rng, 100, 4, 64), _rows("f16", rng, 100, 2, 64)
    p = torch.arange(100, dtype=torch.int32, device=DEV)
    f = ff.ff_rotary_frequencies(32)
    want = ff.ff_rotary(q, k, p, f)
    outs = [torch.zeros_like(x) for x in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ff.ff_rotary(q, k, p, f, q_out=outs[0], k_out=outs[1])
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    p.add_(5)
    want = ff.ff_rotary(q, k, p, f)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
