"""The position-attention oracle against automatic differentiation, differences and the bucket oracle; the frequencies and the refusals
of the entry points, which need no GPU."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import attention as oattn
from oracle import position_attention as opos
from paper_2609_34420_b200 import binding as gt


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_34420_b200 import build
    return build.build()


def tensors(n, H, G, d, seed, spread=1.0):
    rng = np.random.Generator(np.random.PCG64(seed))
    return [rng.standard_normal((n, h, d)) * s for h, s in ((H, spread), (G, 1.0), (G, 1.0), (H, 1.0))]


CASES = [dict(), dict(causal=True), dict(causal=True, prefix=5), dict(causal=True, cap=3.0), dict(cap=2.0),
         dict(causal=True, prefix=9, cap=5.0, slopes=np.array([0.5, 0.25, 0.1, 0.0])), dict(slopes=np.array([1.0, 0.5, 0.0, 2.0]))]


@pytest.mark.parametrize("kw", CASES)
@pytest.mark.parametrize("G", [1, 2, 4])
def test_gradients_against_automatic_differentiation(kw, G):
    q, k, v, do = tensors(13, 4, G, 8, seed=G, spread=3.0)
    r = opos.attention(q, k, v, do, **kw)
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    x = torch.einsum("ihd,jhd->hij", tq, tk.repeat_interleave(4 // G, 1)) / math.sqrt(8)
    if kw.get("cap"):
        x = kw["cap"] * torch.tanh(x / kw["cap"])
    i, j = torch.arange(13)[:, None], torch.arange(13)[None, :]
    if kw.get("slopes") is not None:
        x = x - torch.tensor(kw["slopes"])[:, None, None] * (i - j).abs()
    if kw.get("causal"):
        x = x.masked_fill((j > i) & (j >= kw.get("prefix", 0)), -math.inf)
    o = torch.einsum("hij,jhd->ihd", torch.softmax(x, 2), tv.repeat_interleave(4 // G, 1))
    (o * torch.tensor(do)).sum().backward()
    assert np.allclose(r["out"], o.detach().numpy(), atol=1e-12)
    assert np.allclose(r["lse"], torch.logsumexp(x, 2).detach().numpy(), atol=1e-12)
    for name, t in (("dq", tq), ("dk", tk), ("dv", tv)):
        assert np.allclose(r[name], t.grad.numpy(), atol=1e-11), name


@pytest.mark.parametrize("kw", CASES)
def test_gradients_against_differences(kw):
    q, k, v, do = tensors(7, 4, 2, 4, seed=3)
    r = opos.attention(q, k, v, do, **kw)
    rng = np.random.Generator(np.random.PCG64(9))
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        step = rng.standard_normal(x.shape)
        side = []
        for sign in (1e-5, -1e-5):
            a = {"dq": q, "dk": k, "dv": v} | {name: x + sign * step}
            side.append((opos.attention(a["dq"], a["dk"], a["dv"], **kw)["out"] * do).sum())
        assert abs((side[0] - side[1]) / 2e-5 - (r[name] * step).sum()) < 1e-7


def test_without_options_it_is_the_bucket_form_with_an_empty_table():
    q, k, v, do = tensors(20, 3, 3, 8, seed=5)
    ref = oattn.forward_batch(q, k, v, np.zeros(20 * 32, np.uint8), np.array([0, 640]), np.array([0, 20]), np.zeros((3, 4)))
    r = opos.attention(q, k, v)
    assert np.allclose(r["out"], ref[0], atol=1e-12) and np.allclose(r["lse"], ref[1], atol=1e-12)


@pytest.mark.parametrize("interleaved", [True, False])
def test_rotation_is_a_rotation_and_the_inverse_its_transpose(interleaved):
    rng = np.random.Generator(np.random.PCG64(1))
    x, y = rng.standard_normal((2, 5, 3, 16))
    f, p = np.array([1.0, 0.3, 0.01]), np.array([0, 1, 7, 100, -3])
    rx = opos.rotate(x, f, p, interleaved, 1.5)
    assert np.allclose((rx * y).sum(), (x * opos.rotate(y, f, p, interleaved, 1.5, True)).sum())
    assert np.array_equal(rx[..., 6:], x[..., 6:]) and np.allclose(rx[0, :, :6], 1.5 * x[0, :, :6])
    # scores of rotated rows depend on the difference of positions only
    a, b = opos.rotate(x[:1], f, [3], interleaved), opos.rotate(y[:1], f, [10], interleaved)
    c, e = opos.rotate(x[:1], f, [103], interleaved), opos.rotate(y[:1], f, [110], interleaved)
    assert np.allclose((a * b).sum(2), (c * e).sum(2))


def test_frequencies():
    f = gt.gt_rotary_frequencies(64, 10000.0).numpy()
    assert np.allclose(f, 10000.0 ** (-np.arange(32) / 32), rtol=1e-14)
    assert np.allclose(gt.gt_rotary_frequencies(64, 10000.0, "linear", 4.0).numpy(), f / 4, rtol=1e-14)
    b = gt.gt_rotary_frequencies(64, 10000.0, "base", 4.0).numpy()
    assert np.allclose(b[0], 1.0) and np.allclose(b[-1], f[-1] / 4, rtol=1e-12)      # the slowest pair is slowed by the whole factor
    s = gt.gt_rotary_frequencies(64, 10000.0, "parts", 8.0, 4096, 1.0, 4.0).numpy()
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(s[turns >= 4], f[turns >= 4]) and np.allclose(s[turns <= 1], f[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    assert mid.any() and np.all((s[mid] > f[mid] / 8) & (s[mid] < f[mid]))
    c = (turns[mid] - 1) / 3
    assert np.allclose(s[mid], f[mid] * ((1 - c) / 8 + c), rtol=1e-12)
    assert gt.gt_rotary_frequencies(2).tolist() == [1.0]


@pytest.mark.parametrize("args", [(0,), (3,), (-2,), (8, 0.0), (8, -1.0), (8, math.nan), (8, math.inf), (8, 1e4, "linear", 0.0),
                                  (8, 1e4, "linear", math.nan), (2, 1e4, "base", 2.0), (8, 1e4, "parts", 2.0, 0.0, 1.0, 4.0),
                                  (8, 1e4, "parts", 2.0, 4096, 4.0, 4.0), (8, 1e4, "parts", 2.0, 4096, -1.0, 4.0)])
def test_frequencies_refuse(args):
    with pytest.raises(gt.GtError) as e:
        gt.gt_rotary_frequencies(*args)
    assert e.value.status == 1
    assert gt.lib().gt_rotary_frequencies(8, 1e4, 7, 1.0, 0.0, 0.0, 0.0, (ctypes.c_double * 4)()) == 1
    assert gt.lib().gt_rotary_frequencies(8, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == 1


A = 1 << 20          # stands for a device address: a refused call does not look at it


def batch(T=10, G=1, cu=None, most=None):
    return ctypes.byref(gt._GtBatch(T, G, cu, T if most is None else most))


def fwd(b=None, q=A, k=A, v=A, slopes=None, prefix=None, H=4, G=2, d=64, strides=None, causal=1, cap=0.0, out=A, lse=A, out32=None, ws=A, size=1 << 20):
    return gt.lib().gt_position_attn_fwd(q, k, v, slopes, prefix, b or batch(), H, G, d, strides, causal, cap, out, lse, out32, ws, size, None)


def bwd(b=None, q=A, k=A, v=A, out=A, out32=None, dout=A, lse=A, prefix=None, H=4, G=2, d=64, strides=None, causal=1, cap=0.0, dq=A, dk=A, dv=A,
        ws=A, size=1 << 30):
    return gt.lib().gt_position_attn_bwd(q, k, v, out, out32, dout, lse, None, prefix, b or batch(), H, G, d, strides, causal, cap, dq, dk, dv, ws,
                                         size, None)


def strides(**kw):
    return ctypes.byref(gt._GtRowStrides(**kw))


COMMON = [(dict(b=batch(0)), 1), (dict(b=batch(4, 2)), 1), (dict(b=batch(4, 1, None, 3)), 1), (dict(b=batch(4, 2, A, 5)), 1), (dict(H=0), 1),
          (dict(G=0), 1), (dict(H=4, G=3), 1), (dict(H=2, G=4), 1), (dict(d=48), 2), (dict(d=128), 2), (dict(H=65536, G=1), 2), (dict(cap=-1.0), 1),
          (dict(cap=math.nan), 1), (dict(cap=math.inf), 1), (dict(cap=1e-9), 1), (dict(causal=0, prefix=A), 1), (dict(q=None), 1), (dict(k=None), 1),
          (dict(v=None), 1), (dict(lse=None), 1), (dict(q=A + 8), 1), (dict(k=A + 2), 1), (dict(v=A + 4), 1), (dict(out=A + 8), 1), (dict(out32=A + 4), 1),
          (dict(strides=strides(q=255)), 1), (dict(strides=strides(q=128)), 1), (dict(strides=strides(k=100)), 1), (dict(strides=strides(v=132)), 1),
          (dict(strides=strides(k=-512)), 1), (dict(strides=strides(q=1 << 40)), 1), (dict(ws=None), 3), (dict(ws=A + 8), 3), (dict(size=255), 3)]


@pytest.mark.parametrize("kw,status", COMMON)
def test_attention_refuses(kw, status):
    assert fwd(**kw) == status
    assert bwd(**kw) == status


@pytest.mark.parametrize("kw", [dict(out=None, out32=None), dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dout=A + 8), dict(dq=A + 8),
                                dict(dk=A + 8), dict(dv=A + 8), dict(strides=strides(dq=128)), dict(strides=strides(dk=132)), dict(strides=strides(dv=8))])
def test_backward_refuses(kw):
    assert bwd(**kw) == 1


def test_forward_needs_its_bf16_output():
    assert fwd(out=None, out32=A) == 1


def test_workspaces():
    b = batch(1000, 3, A, 600)
    f = gt.lib().gt_position_attn_fwd_workspace(b, 8, 2, 64)
    w = gt.lib().gt_position_attn_bwd_workspace(b, 8, 2, 64)
    assert f >= 256 + 16 * 3 and w >= 1000 * 8 * (4 * 64 + 32) + 2 * 4 * 1000 * 2 * 64
    assert fwd(b=b, H=8, size=f - 1) == 3 and bwd(b=b, H=8, size=w - 1) == 3
    for bad in ((8, 3, 64), (8, 2, 16), (0, 1, 64)):
        assert gt.lib().gt_position_attn_fwd_workspace(b, *bad) == 0 and gt.lib().gt_position_attn_bwd_workspace(b, *bad) == 0
    assert gt.lib().gt_position_attn_fwd_workspace(batch(0), 8, 2, 64) == 0


def rotary(b=None, q=A, k=A, f=A, p=None, H=4, G=2, d=64, rot=64, dtype=0, sq=0, sk=0, tq=0, tk=0, oq=1 << 24, ok=1 << 25):
    return gt.lib().gt_rotary(q, k, f, p, b or batch(), H, G, d, rot, dtype, 0, 1.0, 0, sq, sk, tq, tk, oq, ok, None)


@pytest.mark.parametrize("kw,status", [(dict(b=batch(0)), 1), (dict(q=None), 1), (dict(oq=None), 1), (dict(f=None), 1), (dict(k=None), 1), (dict(ok=None), 1),
                                       (dict(H=0), 1), (dict(G=-1), 1), (dict(rot=0), 1), (dict(rot=3), 1), (dict(rot=66), 1), (dict(d=48, rot=32), 2),
                                       (dict(d=128), 2), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(sq=255), 1), (dict(sk=-8), 1), (dict(tq=1), 1),
                                       (dict(tk=1 << 40), 1), (dict(q=A + 1), 1), (dict(dtype=2, ok=(1 << 25) + 2), 1), (dict(oq=A, sq=512), 1),
                                       (dict(H=65536), 2), (dict(f=A + 4), 1)])
def test_rotary_refuses(kw, status):
    assert rotary(**kw) == status


def test_bindings_refuse_what_the_library_cannot_see():
    q = torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        gt.gt_rotary(q, None, torch.ones(32, dtype=torch.float64), None, gt.Batch(4), False, 1.0, False, q, None)      # not on the GPU
    with pytest.raises(ValueError):
        gt.gt_rotary(q, q, torch.ones(32, dtype=torch.float64), None, gt.Batch(4), False, 1.0, False, q, None)
    with pytest.raises(ValueError):
        gt.gt_rotary(q, None, torch.ones(32), None, gt.Batch(4), False, 1.0, False, q, None)
    with pytest.raises(ValueError):
        gt.gt_rotary(q.double(), None, torch.ones(32, dtype=torch.float64), None, gt.Batch(4), False, 1.0, False, q.double(), None)
    with pytest.raises(ValueError):
        gt.gt_position_attn_fwd(q, q, q, None, None, gt.Batch(4), True, 0.0, q, torch.zeros(2, 4))


class _OnGpu:
    """A tensor that passes for one on the GPU: a refused call does not look at its memory."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def _bf16(*shape):
    return _OnGpu(torch.zeros(shape, dtype=torch.bfloat16))


@pytest.mark.parametrize("name,wrong", [
    ("k", lambda: _OnGpu(torch.zeros(1, 2, 64, dtype=torch.bfloat16).expand(8, 2, 64))),       # one row for all: would be taken for packed rows
    ("q", lambda: _OnGpu(torch.zeros(8, 1, 64, dtype=torch.bfloat16).expand(8, 4, 64))),
    ("q", lambda: _OnGpu(torch.zeros(2000, dtype=torch.bfloat16).as_strided((8, 4, 64), (192, 64, 1)))),
    ("q", lambda: _bf16(7, 4, 64)), ("k", lambda: _bf16(7, 2, 64)), ("v", lambda: _bf16(8, 1, 64)), ("v", lambda: _bf16(8, 2, 32)), ("out", lambda: _bf16(8, 2, 64)),
    ("lse", lambda: _OnGpu(torch.zeros(4, 7))), ("slopes", lambda: _OnGpu(torch.zeros(2))), ("prefix", lambda: _OnGpu(torch.zeros(0, dtype=torch.int32))),
    ("dq", lambda: _bf16(8, 2, 64)), ("dk", lambda: _bf16(8, 4, 64)), ("dv", lambda: _bf16(4, 2, 64)), ("dout", lambda: _bf16(8, 4, 32)),
    ("out_f32", lambda: _OnGpu(torch.zeros(8, 4, 32)))])
def test_bindings_refuse_tensors_that_are_too_small(name, wrong):
    a = dict(q=_bf16(8, 4, 64), k=_bf16(8, 2, 64), v=_bf16(8, 2, 64), out=_bf16(8, 4, 64), dout=_bf16(8, 4, 64), lse=_OnGpu(torch.zeros(4, 8)),
             slopes=None, prefix=None, batch=gt.Batch(8), causal=True, cap=0.0, dq=_bf16(8, 4, 64), dk=_bf16(8, 2, 64), dv=_bf16(8, 2, 64), out_f32=None,
             workspace=_OnGpu(torch.zeros(256, dtype=torch.uint8)))
    a[name] = wrong()
    with pytest.raises(ValueError):
        gt.gt_position_attn_bwd(**a)
    if name not in ("dout", "dq", "dk", "dv"):
        with pytest.raises(ValueError):
            gt.gt_position_attn_fwd(**{x: a[x] for x in a if x not in ("dout", "dq", "dk", "dv")})


@pytest.mark.parametrize("name,wrong", [("q", lambda: _bf16(7, 4, 64)), ("k", lambda: _OnGpu(torch.zeros(1, 2, 64, dtype=torch.bfloat16).expand(8, 2, 64))),
                                        ("q_out", lambda: _bf16(8, 2, 64)), ("k_out", lambda: _bf16(8, 1, 64)),
                                        ("positions", lambda: _OnGpu(torch.zeros(7, dtype=torch.int32)))])
def test_rotary_binding_refuses_tensors_that_are_too_small(name, wrong):
    a = dict(q=_bf16(8, 4, 64), k=_bf16(8, 2, 64), frequencies=_OnGpu(torch.ones(32, dtype=torch.float64)), positions=None, batch=gt.Batch(8),
             interleaved=False, scale=1.0, inverse=False, q_out=_bf16(8, 4, 64), k_out=_bf16(8, 2, 64))
    a[name] = wrong()
    with pytest.raises(ValueError):
        gt.gt_rotary(**a)


@pytest.mark.parametrize("args", [(8, 1e300, "base", 1e10), (4, 1e4, "base", 1e-200), (8, 1e4, "linear", 1e-310), (8, 1e4, "parts", 1e-310, 4096, 1.0, 4.0)])
def test_frequencies_refuse_what_leaves_the_range(args):
    with pytest.raises(gt.GtError) as e:
        gt.gt_rotary_frequencies(*args)
    assert e.value.status == 1


class _Recorded:
    """Stands for the library: notes the arguments of the last call and succeeds."""

    def __getattr__(self, name):
        def call(*args):
            self.name, self.args = name, args
            return 0
        return call


@pytest.mark.parametrize("f32,ws", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("first", ["workspace", "out_f32", "by name"])
def test_workspace_and_fp32_output_come_in_either_order(monkeypatch, f32, ws, first):
    """Behind the results a call has the workspace, the fp32 output or both."""
    seen = _Recorded()
    monkeypatch.setattr(gt, "lib", lambda: seen)
    monkeypatch.setattr(gt, "_stream", lambda: 0)
    made = _OnGpu(torch.zeros(512, dtype=torch.uint8))
    monkeypatch.setattr(gt, "_workspace", lambda n, device: made)
    t = dict(q=_bf16(8, 4, 64), k=_bf16(8, 2, 64), v=_bf16(8, 2, 64), out=_bf16(8, 4, 64), dout=_bf16(8, 4, 64), lse=_OnGpu(torch.zeros(4, 8)),
             dq=_bf16(8, 4, 64), dk=_bf16(8, 2, 64), dv=_bf16(8, 2, 64))
    out32 = _OnGpu(torch.zeros(8, 4, 64)) if f32 else None
    space = _OnGpu(torch.zeros(1024, dtype=torch.uint8)) if ws else None
    behind = (space, out32) if space is not None else () if out32 is None else (out32,)
    more, named = {"workspace": (behind, {}), "out_f32": ((out32, space), {}), "by name": ((), {"workspace": space, "out_f32": out32})}[first]
    want32, used = out32.data_ptr() if f32 else None, space if ws else made
    got = gt.gt_position_attn_fwd(t["q"], t["k"], t["v"], None, None, gt.Batch(8), True, 0.0, t["out"], t["lse"], *more, **named)
    assert seen.name == "gt_position_attn_fwd" and got is used
    assert seen.args[-6:] == (t["out"].data_ptr(), t["lse"].data_ptr(), want32, used.data_ptr(), used.numel(), 0)
    got = gt.gt_position_attn_bwd(t["q"], t["k"], t["v"], t["out"], t["dout"], t["lse"], None, None, gt.Batch(8), True, 0.0, t["dq"], t["dk"], t["dv"],
                                  *more, **named)
    assert seen.name == "gt_position_attn_bwd" and got is used
    assert seen.args[3:5] == (t["out"].data_ptr(), want32) and seen.args[-3:] == (used.data_ptr(), used.numel(), 0)


@pytest.mark.parametrize("args", [(64, 1e-300, "linear", 1e-100), (64, 1e-300, "parts", 1e-100, 1e-290, 1.0, 8.0)])
def test_frequencies_refuse_a_table_with_an_infinity(args):
    """Base and factor are in range, but not base^-x / factor."""
    with pytest.raises(gt.GtError) as e:
        gt.gt_rotary_frequencies(*args)
    assert e.value.status == 1


def _calls(monkeypatch, **other):
    """One call of each binding on tensors that pass for ones on the GPU, with some replaced; the library only notes what it gets."""
    seen = _Recorded()
    monkeypatch.setattr(gt, "lib", lambda: seen)
    monkeypatch.setattr(gt, "_stream", lambda: 0)
    a = dict(q=_bf16(8, 4, 64), k=_bf16(8, 2, 64), v=_bf16(8, 2, 64), out=_bf16(8, 4, 64), dout=_bf16(8, 4, 64), lse=_OnGpu(torch.zeros(4, 8)),
             slopes=_OnGpu(torch.zeros(4)), prefix=_OnGpu(torch.zeros(1, dtype=torch.int32)), batch=gt.Batch(8), causal=True, cap=0.0, dq=_bf16(8, 4, 64),
             dk=_bf16(8, 2, 64), dv=_bf16(8, 2, 64), out_f32=_OnGpu(torch.zeros(8, 4, 64)), workspace=_OnGpu(torch.zeros(256, dtype=torch.uint8)))
    r = dict(q=a["q"], k=a["k"], frequencies=_OnGpu(torch.ones(32, dtype=torch.float64)), positions=_OnGpu(torch.zeros(8, dtype=torch.int32)),
             batch=a["batch"], interleaved=False, scale=1.0, inverse=False, q_out=_bf16(8, 4, 64), k_out=_bf16(8, 2, 64))
    a, r = a | {x: other[x] for x in other if x in a}, r | {x: other[x] for x in other if x in r}
    fwd = {x: a[x] for x in a if x not in ("dout", "dq", "dk", "dv")}
    return seen, (lambda: gt.gt_position_attn_fwd(**fwd)), (lambda: gt.gt_position_attn_bwd(**a)), (lambda: gt.gt_rotary(**r))


def _on(device, t):
    t.get_device = lambda: device
    return t


@pytest.mark.parametrize("name", ["q", "k", "v", "out", "dout", "lse", "slopes", "prefix", "dq", "dk", "dv", "out_f32", "workspace", "frequencies", "positions",
                                  "q_out", "k_out", "cu_seqlens"])
def test_bindings_refuse_tensors_of_another_device(monkeypatch, name):
    monkeypatch.setattr(gt, "_device", lambda: 1)
    monkeypatch.setattr(_OnGpu, "get_device", lambda self: 1, raising=False)
    monkeypatch.setattr(gt, "_devices", 2)
    seen, *calls = _calls(monkeypatch)
    for call in calls:
        call()
    made = {"lse": _OnGpu(torch.zeros(4, 8)), "slopes": _OnGpu(torch.zeros(4)), "prefix": _OnGpu(torch.zeros(1, dtype=torch.int32)),
            "out_f32": _OnGpu(torch.zeros(8, 4, 64)), "workspace": _OnGpu(torch.zeros(256, dtype=torch.uint8)),
            "frequencies": _OnGpu(torch.ones(32, dtype=torch.float64)), "positions": _OnGpu(torch.zeros(8, dtype=torch.int32))}
    far = _on(0, made.get(name) or _bf16(8, 4 if name in ("q", "out", "dout", "dq", "q_out") else 2, 64))
    if name == "cu_seqlens":
        seen, *calls = _calls(monkeypatch, batch=gt.Batch(8, 1, 8, _on(0, _OnGpu(torch.tensor([0, 8], dtype=torch.int32)))))
    else:
        seen, *calls = _calls(monkeypatch, **{name: far})
    refused = 0
    for call in calls:
        try:
            call()
        except ValueError:
            refused += 1
    both, forward, rotary = ("q", "k", "cu_seqlens"), ("v", "out", "lse", "slopes", "prefix", "out_f32", "workspace"), ("frequencies", "positions", "q_out", "k_out")
    assert refused == (3 if name in both else 2 if name in forward else 1), refused


def test_bindings_refuse_an_lse_with_longer_rows(monkeypatch):
    """Rows behind the batch's belong to q and the results, not to lse, whose heads lie n_total apart."""
    seen, fwd_call, bwd_call, _ = _calls(monkeypatch, lse=_OnGpu(torch.zeros(4, 9)), q=_bf16(9, 4, 64), out=_bf16(9, 4, 64), out_f32=_OnGpu(torch.zeros(9, 4, 64)))
    for call in (fwd_call, bwd_call):
        with pytest.raises(ValueError):
            call()
    seen, fwd_call, bwd_call, _ = _calls(monkeypatch, lse=_OnGpu(torch.zeros(40)))
    fwd_call(), bwd_call()


@pytest.mark.parametrize("cap", [1e-46, -1e-60, 5e-324])
def test_a_cap_that_fp32_takes_for_none_is_out_of_range(monkeypatch, cap):
    assert fwd(cap=math.nan) == 1 and bwd(cap=math.nan) == 1
    seen, fwd_call, bwd_call, _ = _calls(monkeypatch, cap=cap)
    fwd_call()
    assert math.isnan(seen.args[11])
    bwd_call()
    assert math.isnan(seen.args[15])
    seen, fwd_call, bwd_call, _ = _calls(monkeypatch, cap=-0.0)
    fwd_call()
    assert seen.args[11] == 0.0
