"""CPU-only: what ff_attention, ff_attention_backward and ff_rotary refuse, before anything is launched, and the frequencies' table."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import paper_2301_08739_amd as ff
from paper_2301_08739_amd.binding import _AttentionShapeC, _GroupListC, _HeadsC, _RotarySpecC

ARG, UNSUPPORTED, WORKSPACE = -1, -2, -3
H, K, D, N = 4, 2, 16, 100
AT = {name: (i + 1) << 32 for i, name in enumerate(("q", "k", "v", "out", "dout", "dq", "dk", "dv", "lse", "perm", "off", "ws", "pos", "freqs"))}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ff.library_path()):
        pytest.skip("library not built (run __graft_entry__.build())")
    if torch.cuda.is_available():
        pytest.skip("the addresses of these calls are none: only where nothing can be launched")
    return ff.load_library()


def _shape(nq=N, nk=N, G=32, key_G=None, **kw):
    s = _AttentionShapeC(H, K, D, 0.25, None, 4, _GroupListC(AT["perm"], AT["off"], nq, G),
                         _GroupListC(AT["perm"], AT["off"], nk, G if key_G is None else key_G), None)
    for name, v in kw.items():
        setattr(s, name, v)
    return s


def _heads(name, heads, at=None, rs=None, hs=None):
    return _HeadsC(AT[name] if at is None else at, heads * D if rs is None else rs, D if hs is None else hs)


def _forward(lib, s, dtype=1, lse=None, ws=(None, 0), **heads):
    x = {"q": _heads("q", H), "k": _heads("k", K), "v": _heads("v", K), "out": _heads("out", H), **heads}
    return lib.ff_attention(s, *(x[n] for n in ("q", "k", "v", "out")), AT["lse"] if lse is None else lse, dtype, *ws, None)


def _backward(lib, s, dtype=1, lse=AT["lse"], ws=None, **heads):
    x = {n: _heads(n, K if n[-1] in "kv" else H) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")}
    x.update(heads)
    ws = (AT["ws"], lib.ff_attention_backward_workspace_bytes(s, dtype)) if ws is None else ws
    return lib.ff_attention_backward(s, x["q"], x["k"], x["v"], x["out"], lse, *(x[n] for n in ("dout", "dq", "dk", "dv")), dtype, *ws, None)


BAD_SHAPES = [(dict(heads=0), ARG), (dict(kv_heads=0), ARG), (dict(head_dim=0), ARG), (dict(max_groups=-1), ARG), (dict(scale=math.inf), ARG),
              (dict(scale=math.nan), ARG), (dict(kv_heads=3), UNSUPPORTED), (dict(head_dim=129), UNSUPPORTED),
              (dict(queries=_GroupListC(None, None, N, 32)), ARG), (dict(keys=_GroupListC(None, None, N, 32)), ARG),
              (dict(queries=_GroupListC(None, AT["off"], -1, 32)), ARG), (dict(keys=_GroupListC(None, AT["off"], N, 0)), ARG),
              (dict(keys=_GroupListC(None, AT["off"], 1 << 31, 32)), UNSUPPORTED)]


@pytest.mark.parametrize("bad,status", BAD_SHAPES)
def test_shapes(lib, bad, status):
    s = _shape(**bad)
    assert _forward(lib, s) == status
    assert _backward(lib, s, ws=(AT["ws"], 1 << 40)) == status


@pytest.mark.parametrize("bad,status", [(dict(scale=1.5e30), ARG), (dict(scale=-1.5e30), ARG), (dict(max_groups=1 << 28), UNSUPPORTED),
                                        (dict(max_groups=1 << 28, head_dim=128), UNSUPPORTED),
                                        (dict(queries=_GroupListC(None, AT["off"], (1 << 31) - 1, 32)), UNSUPPORTED),
                                        (dict(keys=_GroupListC(None, AT["off"], (1 << 31) - 1, 32)), UNSUPPORTED)])
def test_sizes_that_no_launch_counts(lib, bad, status):
    s, x = _shape(**bad), _wide()
    assert _forward(lib, s, **{n: x[n] for n in ("q", "k", "v", "out")}) == status
    assert _backward(lib, s, ws=(AT["ws"], 1 << 40), **x) == status


def _wide():                                           # heads of up to 128 elements
    return {n: _HeadsC(i << 60, 512, 128) for i, n in enumerate(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), 1)}


def test_rows_that_no_launch_counts(lib):
    assert _backward(lib, _shape(nq=1 << 30, max_groups=1, head_dim=128, G=1 << 20), ws=(AT["ws"], 1 << 50), lse=9 << 60, **_wide()) == UNSUPPORTED
    loose, out = (_HeadsC(1 << 60, 40000, 16) for _ in range(2))   # (in place: heads of 16 elements, 2,048 a row, turned one by one)
    assert lib.ff_rotary(loose, out, 2048, None, None, 0, 1 << 25, 16, AT["pos"], 1, 1, _spec(pairs=7), 1, None) == UNSUPPORTED


def test_workspaces_grow_with_the_rows_that_groups_can_have(lib):
    sizes = []
    for nq in (64, 1 << 24):
        s = _shape(nq=nq, nk=1 << 20, G=4, key_G=1 << 20, max_groups=1)
        sizes.append((lib.ff_attention_workspace_bytes(s, 1), lib.ff_attention_backward_workspace_bytes(s, 1)))
    assert sizes[0][0] == sizes[1][0] > 0
    assert sizes[1][1] - sizes[0][1] == ((1 << 24) - 64) * H * 8   # delta and the start of the scores, of every row


def test_types_and_pointers(lib):
    s = _shape()
    assert _forward(lib, s, dtype=7) == ARG and _backward(lib, s, dtype=-1) == ARG
    assert lib.ff_attention_workspace_bytes(s, 9) == 0 and lib.ff_attention_backward_workspace_bytes(None, 1) == 0
    for name in ("q", "k", "v", "out"):
        assert _forward(lib, s, **{name: None}) == ARG
        assert _forward(lib, s, **{name: _heads(name, H, at=0)}) == ARG
        assert _forward(lib, s, **{name: _heads(name, H, at=AT[name] + 1)}) == ARG       # not on an element's boundary
        assert _forward(lib, s, **{name: _heads(name, H, hs=-1)}) == ARG
    for name in ("dout", "dq", "dk", "dv"):
        assert _backward(lib, s, **{name: None}) == ARG
    assert _backward(lib, s, lse=None) == ARG
    assert _forward(lib, s, lse=AT["lse"] + 2) == ARG


def test_rows_that_share_elements(lib):
    s = _shape()
    assert _forward(lib, s, out=_heads("out", H, rs=H * D - 1)) == ARG                    # rows of the result in each other
    assert _forward(lib, s, out=_heads("out", H, hs=0)) == ARG
    assert _forward(lib, s, out=_heads("out", H, rs=0)) == ARG
    assert _forward(lib, s, out=_heads("q", H)) == ARG                                    # in place
    assert _forward(lib, s, out=_heads("out", H, at=AT["q"] + 2 * D)) == ARG
    assert _forward(lib, s, lse=AT["out"] + 4) == ARG
    assert _backward(lib, s, dk=_heads("dv", K)) == ARG
    assert _backward(lib, s, dq=_heads("dout", H)) == ARG
    # parts of one packed array lie beside each other; one element further they meet
    width = 2 * (H + 2 * K) * D
    at = AT["dq"]
    packed = dict(dq=_heads("dq", H, at=at, rs=width), dk=_heads("dk", K, at=at + 2 * H * D, rs=width), dv=_heads("dv", K, at=at + 2 * (H + K) * D, rs=width))
    meets = dict(packed, dk=_heads("dk", K, at=at + 2 * H * D - 2, rs=width))
    assert _backward(lib, s, **meets) == ARG
    few = _shape(nq=2, nk=1 << 20, G=1, key_G=1 << 20, max_groups=2)
    assert _backward(lib, few, **packed, ws=(at, 1 << 40)) == ARG                        # the workspace in the gradients
    assert _backward(lib, s, dq=_heads("dq", H, at=AT["perm"])) == ARG
    assert _forward(lib, s, out=_heads("out", H, at=AT["off"])) == ARG


def test_workspaces(lib):
    few = _shape(nq=2, nk=1 << 20, G=1, key_G=1 << 20, max_groups=2)
    for run, need in ((_forward, lib.ff_attention_workspace_bytes(few, 1)), (_backward, lib.ff_attention_backward_workspace_bytes(few, 1))):
        assert need > 0
        for ws in ((None, 0), (AT["ws"], need - 1), (AT["ws"] + 128, need)):
            assert run(lib, few, ws=ws) == WORKSPACE


def test_empty_calls_launch_nothing(lib):
    assert _forward(lib, _shape(nq=0, nk=0)) == 0
    assert _forward(lib, _shape(max_groups=0)) == 0
    assert _backward(lib, _shape(nq=0, nk=0)) == 0


def _rotary(lib, spec=None, n=N, head_dim=D, dtype=1, q=None, q_out=None, k=None, k_out=None, K=K, pos=AT["pos"], strides=(1, 1)):
    spec = _spec() if spec is None else spec
    both = K > 0
    return lib.ff_rotary(q or _heads("q", H), q_out or _heads("out", H), H, k or (_heads("k", K) if both else None),
                         k_out or (_heads("dk", K) if both else None), K, n, head_dim, pos, *strides, spec, dtype, None)


def _spec(axes=1, pairs=8, layout=0, inverse=0, amplitude=1.0, freqs=AT["freqs"]):
    return _RotarySpecC(axes, pairs, layout, inverse, amplitude, freqs)


@pytest.mark.parametrize("bad,status", [(dict(axes=0), ARG), (dict(pairs=0), ARG), (dict(layout=2), ARG), (dict(inverse=2), ARG), (dict(amplitude=math.nan), ARG),
                                        (dict(freqs=None), ARG), (dict(freqs=AT["freqs"] + 4), ARG), (dict(axes=4, pairs=1), UNSUPPORTED),
                                        (dict(pairs=9), UNSUPPORTED), (dict(axes=2, pairs=1 << 30), UNSUPPORTED)])
def test_rotary_specs(lib, bad, status):
    assert _rotary(lib, _spec(**bad)) == status


def test_rotary_arguments(lib):
    assert _rotary(lib, n=0) == 0
    assert _rotary(lib, dtype=3) == ARG and _rotary(lib, n=-1) == ARG and _rotary(lib, pos=None) == ARG and _rotary(lib, pos=AT["pos"] + 2) == ARG
    assert _rotary(lib, strides=(-1, 1)) == ARG
    assert _rotary(lib, head_dim=257) == UNSUPPORTED
    assert _rotary(lib, q_out=_heads("q", H, at=AT["q"] + 2)) == ARG                       # neither in place nor beside
    assert _rotary(lib, q_out=_heads("q", H, rs=H * D + 8)) == ARG
    assert _rotary(lib, q_out=_heads("dk", H)) == ARG                                      # where k's result goes
    assert _rotary(lib, q_out=_heads("out", H, at=AT["pos"])) == ARG
    assert _rotary(lib, q_out=_heads("out", H, at=AT["freqs"] - 32)) == ARG
    assert _rotary(lib, K=0, k=_heads("k", 2)) == ARG


def test_frequencies():
    if not os.path.exists(ff.library_path()):
        pytest.skip("library not built")
    f = ff.ff_rotary_frequencies(5, axes=2, base=100.0, device="cpu")
    want = 100.0 ** (-np.arange(5) / 5)
    assert f.shape == (2, 5) and np.allclose(f[1].numpy(), want, rtol=1e-14)
    assert np.allclose(ff.ff_rotary_frequencies(5, base=100.0, factor=4.0, device="cpu")[0].numpy(), want / 4, rtol=1e-14)
    long = ff.ff_rotary_frequencies(64, factor=8.0, original_length=8192, device="cpu")[0].numpy()
    plain = 10000.0 ** (-np.arange(64) / 64)
    turns = 8192 * plain / (2 * np.pi)
    assert np.allclose(long[turns >= 32], plain[turns >= 32]) and np.allclose(long[turns <= 1], plain[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 32)
    w = (turns[mid] - 1) / 31
    assert mid.any() and np.allclose(long[mid], plain[mid] * (w + (1 - w) / 8))
    for bad in (dict(pairs=0), dict(pairs=4, base=0.0), dict(pairs=4, factor=-1.0), dict(pairs=4, original_length=-1.0), dict(pairs=4, low_turns=3.0, high_turns=3.0)):
        with pytest.raises(ff.FlatformerError):
            ff.ff_rotary_frequencies(**bad, device="cpu")


def test_the_binding_refuses_tensors_that_do_not_fit():
    if not os.path.exists(ff.library_path()):
        pytest.skip("library not built")
    r = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    ok = dict(q=r(8, 4, 16), k=r(8, 2, 16), v=r(8, 2, 16), perm=i32(8), group_offsets=i32(3), num_groups=i32(1), max_groups=2, G=4)
    bad = [dict(q=r(8, 64)), dict(q=r(8, 4, 16, dt=torch.float64)), dict(k=r(8, 2, 8)), dict(v=r(8, 2, 16, dt=torch.bfloat16)), dict(v=r(7, 2, 16)),
           dict(q=r(8, 16, 4).transpose(1, 2)), dict(perm=i32(7)), dict(perm=torch.zeros(8, dtype=torch.int64)), dict(group_offsets=i32(2)),
           dict(group_offsets=None), dict(num_groups=torch.zeros(1)), dict(key_mask=torch.ones(8)), dict(key_mask=torch.ones(7, dtype=torch.bool)),
           dict(key_perm=i32(8)), dict(k=r(9, 2, 16), v=r(9, 2, 16)), dict(key_offsets=i32(2))]
    for change in bad:
        with pytest.raises(ff.FlatformerError):
            ff.ff_attention(**dict(ok, **change))
        with pytest.raises(ff.FlatformerError):
            ff.ff_attention_backward(**dict(ok, **change), out=r(8, 4, 16), lse=r(8, 4), dout=r(8, 4, 16))
    with pytest.raises(ff.FlatformerError, match="GPU"):
        ff.ff_attention(**ok)
    with pytest.raises(ff.FlatformerError, match="lse"):
        ff.ff_attention_backward(**ok, out=r(8, 4, 16), lse=None, dout=r(8, 4, 16))
    f = torch.zeros(1, 4, dtype=torch.float64)
    for change in (dict(positions=torch.zeros(8, dtype=torch.int64)), dict(positions=i32(7)), dict(freqs=f.float()), dict(freqs=f[0]), dict(k=r(8, 16)),
                   dict(freqs=f.expand(2, 4))):
        with pytest.raises(ff.FlatformerError):
            ff.ff_rotary(**dict(dict(q=ok["q"], k=ok["k"], positions=i32(8), freqs=f), **change))
