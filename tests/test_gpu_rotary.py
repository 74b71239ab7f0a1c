"""gt_rotary against the oracle.  A result is off by the angle (5e-7 rad at the farthest, 2^-24 of a turn from the reduction's rounding to
fp32), sine and cosine (2 units in the last place), two products and a sum in fp32 (2^-24 each), and its own rounding, half a step."""
import numpy as np
import pytest
import torch

from oracle import position_attention as opos
from paper_2609_34420_b200 import binding as gt

from gpu_util import to_f64

pytestmark = pytest.mark.gpu
LEFT = 55.0
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SLIP = 5e-7 + 2 ** -24 * 2 * np.pi + 2 * 2 ** -23 + 4 * 2 ** -24


def limit(x, y, frequencies, interleaved, scale, dtype):
    """|a| + |b| of an element's pair times what the rotation may be off, and the rounding; 0 for the channels that are not rotated."""
    half, size = len(frequencies), np.abs(x)
    r = np.zeros_like(size)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    r[..., a] = r[..., b] = (size[..., a] + size[..., b]) * scale * SLIP
    r[..., :2 * half] += np.abs(y[..., :2 * half]) * torch.finfo(dtype).eps / 2 * 1.001 + (2.0 ** -25 if dtype == torch.float16 else 0)
    return r


def check(x, y, f, positions, interleaved, scale, inverse):
    ref = opos.rotate(to_f64(x), f.numpy(), positions, interleaved, scale, inverse)
    off = np.abs(to_f64(y) - ref)
    assert np.all(off <= limit(to_f64(x), ref, f, interleaved, scale, x.dtype)), float(off.max())


def make(T, H, G, d, dtype, seed=0):
    rng = np.random.Generator(np.random.PCG64(seed))
    return [torch.from_numpy(rng.standard_normal((T, h, d))).to(dtype).cuda() for h in (H, G)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("d,rot", [(32, 32), (32, 16), (32, 2), (32, 10), (64, 64), (64, 32), (64, 16), (64, 8), (64, 24), (64, 2), (64, 62)])
def test_types_layouts_and_widths(dtype, interleaved, d, rot):
    q, k = make(37, 5, 2, d, TYPES[dtype], rot)
    f = gt.gt_rotary_frequencies(rot, 10000.0)
    oq, ok = torch.full_like(q, LEFT), torch.full_like(k, LEFT)
    for inverse in (False, True):
        gt.gt_rotary(q, k, f.cuda(), None, gt.Batch(37), interleaved, 1.25, inverse, oq, ok)
        check(q, oq, f, np.arange(37), interleaved, 1.25, inverse)
        check(k, ok, f, np.arange(37), interleaved, 1.25, inverse)
        assert torch.equal(oq[..., rot:], q[..., rot:]) and torch.equal(ok[..., rot:], k[..., rot:])


@pytest.mark.parametrize("T", [1, 2, 7, 8, 31, 33, 500, 5000])
@pytest.mark.parametrize("H,G", [(1, 0), (1, 1), (7, 1), (16, 4), (40, 8), (130, 1)])
def test_rows_and_heads(T, H, G):
    q, k = make(T, H, max(G, 1), 64, torch.bfloat16, T)
    f = gt.gt_rotary_frequencies(32)
    oq, ok = torch.full_like(q, LEFT), torch.full_like(k, LEFT)
    gt.gt_rotary(q, k if G else None, f.cuda(), None, gt.Batch(T), False, 1.0, False, oq, ok if G else None)
    check(q, oq, f, np.arange(T), False, 1.0, False)
    if G:
        check(k, ok, f, np.arange(T), False, 1.0, False)
    else:
        assert bool((ok == LEFT).all())


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("rot", [64, 6])
def test_far_positions(interleaved, rot):
    position = np.array([0, 1, -1, 1 << 20, (1 << 20) + 1, (1 << 31) - 1, -(1 << 31), 123456789, 16777217], np.int64)
    q, k = make(len(position), 3, 1, 64, torch.float32, 3)
    f = gt.gt_rotary_frequencies(rot, 500000.0)
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    p = torch.from_numpy(position.astype(np.int32)).cuda()
    gt.gt_rotary(q, k, f.cuda(), p, gt.Batch(len(position)), interleaved, 1.0, False, oq, ok)
    check(q, oq, f, position, interleaved, 1.0, False)
    check(k, ok, f, position, interleaved, 1.0, False)


@pytest.mark.parametrize("rot", [64, 6])
@pytest.mark.parametrize("lengths", [[3, 0, 0, 200, 1, 1, 0, 77, 0], [0, 0, 1], [1] * 100, [5] + [0] * 70 + [40] * 3])
def test_documents_and_rows_behind_the_last_one(rot, lengths):
    n, extra = sum(lengths), 19
    q, k = make(n + extra, 4, 2, 64, torch.bfloat16, n)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device="cuda")
    f = gt.gt_rotary_frequencies(rot)
    oq, ok = torch.full_like(q, LEFT), torch.full_like(k, LEFT)
    batch = gt.Batch(n + extra, len(lengths), max(lengths), cu)
    gt.gt_rotary(q, k, f.cuda(), None, batch, True, 1.0, False, oq, ok)
    position = np.concatenate([np.arange(x) for x in lengths])
    check(q[:n], oq[:n], f, position, True, 1.0, False)
    check(k[:n], ok[:n], f, position, True, 1.0, False)
    assert bool((oq[n:] == LEFT).all()) and bool((ok[n:] == LEFT).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lead", [0, 1, 3])
@pytest.mark.parametrize("interleaved", [True, False])
def test_parts_of_a_projection_in_place_and_at_any_address(dtype, lead, interleaved):
    T, H, G, d, rot = 45, 4, 2, 32, 16
    rng = np.random.Generator(np.random.PCG64(lead))
    flat = torch.from_numpy(rng.standard_normal(lead + T * ((H + 2 * G) * d + lead))).to(TYPES[dtype]).cuda()
    rows = flat[lead:].view(T, -1)
    q, k, rest = rows[:, :H * d].unflatten(1, (H, d)), rows[:, H * d:(H + G) * d].unflatten(1, (G, d)), rows[:, (H + G) * d:]
    before = q.clone(), k.clone(), rest.clone()
    f = gt.gt_rotary_frequencies(rot)
    oq, ok = torch.empty_like(before[0]), torch.empty_like(before[1])
    gt.gt_rotary(q, k, f.cuda(), None, gt.Batch(T), interleaved, 1.0, False, oq, ok)
    check(before[0], oq, f, np.arange(T), interleaved, 1.0, False)
    gt.gt_rotary(q, k, f.cuda(), None, gt.Batch(T), interleaved, 1.0, False, q, k)
    assert torch.equal(q, oq) and torch.equal(k, ok) and torch.equal(rest, before[2])


def test_values_that_are_not_rotated_pass_through_as_they_are():
    q = torch.full((4, 2, 64), float("inf"), dtype=torch.bfloat16, device="cuda")
    q[..., :16] = 1.0
    q[..., 40] = float("nan")
    for interleaved in (True, False):
        out = torch.empty_like(q)
        gt.gt_rotary(q, None, gt.gt_rotary_frequencies(16).cuda(), None, gt.Batch(4), interleaved, 2.0, False, out, None)
        assert bool(out[..., :16].isfinite().all()) and torch.equal(out[..., 16:].view(torch.int16), q[..., 16:].view(torch.int16))


def test_captured_on_another_stream_and_replayed():
    q, k = make(100, 4, 2, 64, torch.bfloat16, 1)
    f, p = gt.gt_rotary_frequencies(64), torch.arange(100, dtype=torch.int32, device="cuda")
    fd, oq, ok = f.cuda(), torch.empty_like(q), torch.empty_like(k)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gt.gt_rotary(q, k, fd, p, gt.Batch(100), False, 1.0, False, oq, ok)
    p += 1000
    g.replay()
    torch.cuda.synchronize()
    check(q, oq, f, np.arange(100) + 1000, False, 1.0, False)
    check(k, ok, f, np.arange(100) + 1000, False, 1.0, False)


@pytest.mark.parametrize("rot", [64, 6])
def test_offsets_beyond_32_bits(rot):
    T, H = 530000, 64
    q = torch.zeros(T, H, 64, dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 1 << 31
    q[-9:] = make(9, H, 1, 64, torch.bfloat16, 2)[0]
    f, out = gt.gt_rotary_frequencies(rot), torch.empty_like(q)
    gt.gt_rotary(q, None, f.cuda(), None, gt.Batch(T), True, 1.0, False, out, None)
    check(q[-9:], out[-9:], f, np.arange(T - 9, T), True, 1.0, False)
    assert not out[:-9].any()


@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("rot", [64, 6])
def test_far_positions_within_the_derived_error_of_their_angles(interleaved, rot):
    """The angle w is off by 3 x 2^-53 w (three roundings in fp64) and, reduced to half a turn at most, by 2^-25 pi (its rounding to fp32); sine and
    cosine by two units in the last place, 2 x 2^-24; then two products and a sum, 2^-24 each of no more than |a| + |b|."""
    rng = np.random.Generator(np.random.PCG64(5))
    position = np.concatenate([[0, 1, -1, (1 << 31) - 1, -(1 << 31)], rng.integers(-(1 << 31), 1 << 31, 300), rng.integers(0, 1 << 20, 300)])
    T, d = len(position), 64
    q, k = make(T, 2, 1, d, torch.float32, 4)
    f = gt.gt_rotary_frequencies(rot, 500000.0)
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    p = torch.from_numpy(position.astype(np.int32)).cuda()
    gt.gt_rotary(q, k, f.cuda(), p, gt.Batch(T), interleaved, 1.0, False, oq, ok)
    angle = np.abs(position[:, None] * f.numpy()[None, :])
    slip = 3 * 2.0 ** -53 * angle + 2.0 ** -25 * np.pi + 2 * 2.0 ** -24 + 3 * 2.0 ** -24
    for x, y in ((q, oq), (k, ok)):
        x, y = to_f64(x), to_f64(y)
        off = np.abs(y - opos.rotate(x, f.numpy(), position, interleaved))
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        limit = (np.abs(x[..., a]) + np.abs(x[..., b])) * slip[:, None, :]
        assert np.all(off[..., a] <= limit) and np.all(off[..., b] <= limit), float(max((off[..., a] / limit).max(), (off[..., b] / limit).max()))
