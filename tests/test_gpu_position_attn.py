"""gt_position_attn_fwd / gt_position_attn_bwd against the fp64 oracle, through the C ABI.

Elementwise, a result may be off by what the oracle derives from half a step of every rounding to bf16; as a whole (2-norm) by what it
derives from independent roundings, and 10 % for the sample that a result of 4 096 values or more is."""
import numpy as np
import pytest
import torch

from oracle import position_attention as opos
from paper_2609_34420_b200 import binding as gt

from gpu_util import rel_l2, to_f64

pytestmark = pytest.mark.gpu
ONE = 2.0 ** -8 / 3 ** 0.5
WHOLE = ("out", "dq", "dk", "dv")
LEFT = 77.0          # what lies in results before a call


class Case:
    def __init__(self, lengths, H=4, G=2, d=64, causal=True, prefix=None, slopes=None, cap=0.0, spread=1.0, shift=0.0, extra=0, seed=0, apart=False):
        rng = np.random.Generator(np.random.PCG64(seed))
        dev = "cuda"
        self.cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        self.n, T = int(self.cu[-1]), int(self.cu[-1]) + extra
        self.T, self.H, self.G, self.d, self.causal, self.cap = T, H, G, d, causal, cap

        def normal(h, std=1.0):
            return torch.from_numpy(rng.standard_normal((T, h, d)) * std).bfloat16().to(dev)

        q, k, v, self.dout = normal(H, spread), normal(G), normal(G), normal(H)
        if shift:                        # every score moves by about `shift`
            q[:, :, 0], k[:, :, 0] = 8.0, shift
        if apart:
            rows = torch.full((T, H + 2 * G + 1, d), LEFT, dtype=torch.bfloat16, device=dev)
            self.q, self.k, self.v = rows[:, :H], rows[:, H:H + G], rows[:, H + G:H + 2 * G]
            self.q[:], self.k[:], self.v[:] = q, k, v
            grads = torch.full_like(rows, LEFT)
            self.dq, self.dk, self.dv = grads[:, :H], grads[:, H:H + G], grads[:, H + G:H + 2 * G]
            self.gap = grads[:, H + 2 * G:]
        else:
            self.q, self.k, self.v = q, k, v
            self.dq, self.dk, self.dv = (torch.full_like(x, LEFT) for x in (q, k, v))
            self.gap = None
        many = len(lengths) > 1 or extra
        self.batch = gt.Batch(T, len(lengths), T if len(lengths) == 1 else max(1, *lengths), torch.from_numpy(self.cu).to(dev) if many else None)
        self.prefix = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=dev)
        self.slopes = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device=dev)
        self.out = torch.full((T, H, d), LEFT, dtype=torch.bfloat16, device=dev)
        self.out32 = torch.full((T, H, d), LEFT, device=dev)
        self.lse = torch.full((H, T), LEFT, device=dev)

    def forward(self, exact=True, ws=None):
        return gt.gt_position_attn_fwd(self.q, self.k, self.v, self.slopes, self.prefix, self.batch, self.causal, self.cap, self.out, self.lse,
                                       self.out32 if exact else None, ws)

    def backward(self, exact=True, ws=None):
        return gt.gt_position_attn_bwd(self.q, self.k, self.v, self.out, self.dout, self.lse, self.slopes, self.prefix, self.batch, self.causal,
                                       self.cap, self.dq, self.dk, self.dv, self.out32 if exact else None, ws)

    def oracle(self):
        n = self.n
        q, k, v, do = (to_f64(x)[:n] for x in (self.q, self.k, self.v, self.dout))
        return opos.batch_attention(q, k, v, do, self.cu, self.causal, None if self.prefix is None else self.prefix.tolist(),
                                    None if self.slopes is None else to_f64(self.slopes), self.cap)

    def results(self):
        return {"out": to_f64(self.out), "lse": to_f64(self.lse), "dq": to_f64(self.dq), "dk": to_f64(self.dk), "dv": to_f64(self.dv)}

    def check(self, exact=True, ref=None, names=("out", "lse", "dq", "dk", "dv")):
        ref, got, n = ref or self.oracle(), self.results(), self.n
        for name in names:
            x = got[name][:, :n] if name == "lse" else got[name][:n]
            limit = ref["bounds"][name if exact or name not in ("dq", "dk") else name + "_out"]
            off = np.abs(x - ref[name])
            assert np.all(off <= limit), (name, float((off / limit).max()), np.argwhere(~(off <= limit))[:4].tolist())
            if name in WHOLE and (exact or name not in ("dq", "dk")) and x.size >= 4096:
                assert np.linalg.norm(x - ref[name]) <= 1.1 * ref["norms"][name], (name, float(np.linalg.norm(x - ref[name]) / ref["norms"][name]))
            behind = got[name][:, n:] if name == "lse" else got[name][n:]
            assert np.all(behind == LEFT), name
        assert self.gap is None or bool((self.gap == LEFT).all())
        return ref

    def run(self, exact=True):
        self.forward_ws = self.forward(exact)
        gt.gt_check(self.forward_ws)
        gt.gt_check(self.backward(exact))
        return self.check(exact)


@pytest.mark.parametrize("n", [1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 300, 384, 385, 513])
@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths(n, d, causal):
    Case([n], H=2, G=1, d=d, causal=causal, seed=n).run()


@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (4, 1), (6, 2), (8, 4), (12, 4)])
def test_heads(H, G):
    Case([200], H=H, G=G, seed=H).run()


OPTIONS = [dict(), dict(cap=5.0, spread=3.0), dict(slopes=True), dict(prefix=True), dict(prefix=True, slopes=True, cap=20.0, spread=6.0),
           dict(causal=False, slopes=True), dict(causal=False, cap=2.0, spread=4.0), dict(causal=False, slopes=True, cap=50.0, spread=2.0),
           dict(spread=15.0), dict(spread=15.0, slopes=True), dict(cap=30.0, spread=25.0), dict(shift=30.0), dict(shift=-30.0),
           dict(shift=-30.0, causal=False, slopes=True), dict(cap=50.0, shift=-30.0), dict(cap=1e-3), dict(cap=1e6)]


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("lengths", [[600], [1, 130, 0, 300, 5, 0, 256, 128, 7], [0, 0, 129, 384, 0]])
@pytest.mark.parametrize("d", [32, 64])
def test_options(options, lengths, d):
    o = dict(options)
    if o.pop("slopes", False):
        o["slopes"] = [0.5, 0.0625, 0.0, 2.0]
    if o.pop("prefix", False):
        o["prefix"] = [[9, 200, -5, 1 << 30, 3, 0, 129, 128, -(1 << 31)][i % 9] for i in range(len(lengths))]
    Case(lengths, d=d, seed=len(lengths), **o).run()


@pytest.mark.parametrize("prefix", [1, 64, 127, 128, 129, 255, 256, 257, 299, 300, 301])
def test_prefixes_at_the_edges_of_tiles(prefix):
    Case([300], H=2, G=2, prefix=[prefix], slopes=[0.1, 1.0], seed=prefix).run()
    Case([700, 300, 520], H=2, G=2, prefix=[prefix] * 3, seed=prefix).run()


@pytest.mark.parametrize("exact", [True, False])
def test_rows_apart_and_rows_behind_the_last_document(exact):
    Case([100, 0, 257, 60], H=4, G=2, cap=10.0, spread=2.0, extra=150, apart=True, seed=1).run(exact)
    Case([300], H=4, G=4, extra=1, apart=True, seed=2).run(exact)
    empty = Case([0, 0], H=2, G=1, extra=3)
    gt.gt_check(empty.forward(exact))
    gt.gt_check(empty.backward(exact))
    assert all((x == LEFT).all() for x in empty.results().values())


def test_without_the_fp32_output_peaked_rows_stay_within_their_bounds():
    Case([400, 33], H=4, G=4, spread=6.0, seed=5).run(exact=False)


def test_large_blocks_of_two_tiles_and_the_work_list():
    """Enough documents for blocks of two query tiles and, in the backward, the list of the work."""
    rng = np.random.Generator(np.random.PCG64(3))
    Case([int(n) for n in rng.integers(0, 700, 24)], H=8, G=2, prefix=[int(n) for n in rng.integers(0, 300, 24)], slopes=list(2.0 ** -np.arange(1, 9)),
         cap=30.0, spread=3.0, seed=4).run()
    Case([int(n) for n in rng.integers(1, 90, 70)] + [1000], H=8, G=8, seed=6).run()


def test_many_documents_of_very_different_lengths():
    lengths = [1200] + [5] * 300
    Case(lengths, H=4, G=4, d=32, seed=8).run()


@pytest.mark.parametrize("causal", [True, False])
def test_other_documents_values_do_not_leak(causal):
    """NaN and infinities in the rows of another document, and behind the last one, change nothing."""
    kw = dict(lengths=[70, 200, 300], H=4, G=2, causal=causal, extra=40, seed=11)
    clean = Case(**kw)
    clean.run()
    for bad in (float("nan"), float("inf")):
        c = Case(**kw)
        for x in (c.q, c.k, c.v, c.dout):
            x[70:270] = bad
            x[570:] = -bad
        gt.gt_check(c.forward())
        c.lse[:, 70:270] = bad
        c.out32[70:270] = bad
        gt.gt_check(c.backward())
        for rows in (slice(0, 70), slice(270, 570)):
            assert torch.equal(c.out[rows], clean.out[rows]) and torch.equal(c.lse[:, rows], clean.lse[:, rows])
            for name in ("dq", "dk", "dv"):
                x, y = to_f64(getattr(c, name)[rows]), to_f64(getattr(clean, name)[rows])
                assert np.isfinite(x).all() and rel_l2(x, y) <= 2 * ONE, name              # (the order of the sums)
        assert bool((c.out[570:] == LEFT).all()) and bool((c.dk[570:] == LEFT).all())


def test_keys_that_no_query_may_see_yet_do_not_matter():
    """Large finite values in the future of a causal row stay without effect."""
    c = Case([256], H=2, G=2, seed=12)
    c.run()
    ref = to_f64(c.out)[:128]
    c.k[128:], c.v[128:] = 300.0, -300.0
    gt.gt_check(c.forward())
    assert np.array_equal(to_f64(c.out)[:128], ref)


def test_another_stream():
    c = Case([500, 300], H=4, G=2, seed=13)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a, b = c.forward(), c.backward()
        gt.gt_check(a)
        gt.gt_check(b)
    c.check()


def test_captured_and_replayed():
    c = Case([400, 300], H=4, G=2, prefix=[10, 200], seed=14)
    wf, wb = c.forward(), c.backward()
    gt.gt_check(wb)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward(ws=wf)
        c.backward(ws=wb)
    other = Case([400, 300], H=4, G=2, prefix=[10, 200], seed=15)
    for x in ("q", "k", "v", "dout"):
        getattr(c, x).copy_(getattr(other, x))
    for _ in range(2):
        for x in (c.out, c.out32, c.lse, c.dq, c.dk, c.dv):
            x.fill_(LEFT)
        g.replay()
        gt.gt_check(wf)
        gt.gt_check(wb)
        c.check()


def test_the_same_call_twice_and_one_workspace_for_both_directions():
    c = Case([333, 64, 1], H=4, G=1, slopes=[0.1] * 4, seed=16)
    size = max(gt.gt_position_attn_fwd_workspace(c.batch, 4, 1, 64), gt.gt_position_attn_bwd_workspace(c.batch, 4, 1, 64))
    ws = gt._workspace(size, "cuda")
    ref = None
    for _ in range(3):
        c.forward(ws=ws)
        c.backward(ws=ws)
        gt.gt_check(ws)
        ref = c.check(ref=ref)


def test_forward_is_the_same_from_run_to_run():
    c = Case([777], H=8, G=8, cap=10.0, seed=17)
    c.forward()
    first = c.out.clone(), c.lse.clone(), c.out32.clone()
    c.forward()
    assert all(torch.equal(a, b) for a, b in zip(first, (c.out, c.lse, c.out32)))


def test_fp32_output():
    c = Case([300, 20], H=4, G=2, spread=4.0, seed=18)
    ref = c.run()
    off = np.abs(to_f64(c.out32)[:320] - ref["out"])
    assert np.all(off <= ref["bounds"]["out"])
    assert np.linalg.norm(to_f64(c.out32) - ref["out"]) <= 1.1 * ref["norms"]["out"]
    assert torch.equal(c.out32.bfloat16(), c.out)


def test_one_key_gives_exactly_its_value():
    c = Case([1, 1, 1], H=4, G=4, seed=19)
    c.run()
    assert torch.equal(c.out, c.v) and torch.equal(c.out32, c.v.float()) and torch.equal(c.dv, c.dout)


def test_offsets_beyond_32_bits():
    """q and out of more than 2^31 elements; the last documents."""
    n, docs, H, d = 40, 13200, 64, 64
    T = n * docs
    assert T * H * d > 1 << 31
    q = torch.zeros(T, H, d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    last = slice(T - 3 * n, T)
    q[last] = torch.randn(3 * n, H, d, device="cuda", generator=g).bfloat16()
    k, v = (torch.randn(T, 1, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    cu = torch.arange(docs + 1, device="cuda", dtype=torch.int32) * n
    out, lse = torch.empty_like(q), torch.empty(H, T, device="cuda")
    batch = gt.Batch(T, docs, n, cu)
    ws = gt.gt_position_attn_fwd(q, k, v, None, None, batch, True, 0.0, out, lse)
    gt.gt_check(ws)
    ref = opos.batch_attention(to_f64(q[last]), to_f64(k[last]), to_f64(v[last]), None, np.arange(4) * n, True)
    assert np.all(np.abs(to_f64(out[last]) - ref["out"]) <= ref["bounds"]["out"])
    assert np.all(np.abs(to_f64(lse[:, last]) - ref["lse"]) <= ref["bounds"]["lse"])
    dout = torch.zeros_like(q)
    dout[last] = torch.randn(3 * n, H, d, device="cuda", generator=g).bfloat16()
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    gt.gt_check(gt.gt_position_attn_bwd(q, k, v, out, dout, lse, None, None, batch, True, 0.0, dq, dk, dv))
    ref = opos.batch_attention(to_f64(q[last]), to_f64(k[last]), to_f64(v[last]), to_f64(dout[last]), np.arange(4) * n, True)
    for name, x in (("dq", dq), ("dk", dk), ("dv", dv)):
        off = "" if name == "dv" else "_out"
        assert np.all(np.abs(to_f64(x[last]) - ref[name]) <= ref["bounds"][name + off]), name
    assert not dq[:last.start].any() and not dv[:last.start].any()


def test_layer_with_rotary_positions():
    """Rotation, attention and their gradients in a row, as a layer uses them, against the oracle of the whole."""
    lengths, H, G, d, rot = [300, 1, 150], 4, 2, 64, 32
    c = Case(lengths, H=H, G=G, d=d, cap=20.0, spread=2.0, seed=20)
    f = gt.gt_rotary_frequencies(rot, 10000.0, "parts", 4.0, 100, 1.0, 8.0)
    fd = f.cuda()
    q0, k0 = c.q.clone(), c.k.clone()
    gt.gt_rotary(c.q, c.k, fd, None, c.batch, False, 1.1, False, c.q, c.k)              # in place
    ref = c.run()
    position = np.concatenate([np.arange(n) for n in lengths])
    for x, x0 in ((c.q, q0), (c.k, k0)):
        y = opos.rotate(to_f64(x0), f.numpy(), position, False, 1.1)
        assert np.all(np.abs(to_f64(x) - y) <= 2.0 ** -8 * np.abs(y) + 1e-6 * np.abs(to_f64(x0)).max())
    dq, dk = torch.empty_like(c.dq), torch.empty_like(c.dk)
    gt.gt_rotary(c.dq, c.dk, fd, None, c.batch, False, 1.1, True, dq, dk)
    for name, x in (("dq", dq), ("dk", dk)):
        y = opos.rotate(ref[name], f.numpy(), position, False, 1.1, True)
        assert np.linalg.norm(to_f64(x) - y) <= 1.1 * 1.1 * ref["norms"][name] + ONE * np.linalg.norm(y), name          # (turned and scaled by 1.1, rounded once more)


def test_results_at_any_16_byte_address():
    """Results that begin in the middle of a sector; q, k and v, too."""
    c = Case([200, 77], H=4, G=4, d=32, seed=21)

    def moved(x):
        return torch.cat([x.new_zeros(8), x.flatten()])[8:].view_as(x)

    for name in ("q", "k", "v", "dout", "out", "dq", "dk", "dv"):
        setattr(c, name, moved(getattr(c, name)))
        assert getattr(c, name).data_ptr() % 32 == 16
    c.out32 = torch.cat([c.out32.new_zeros(4), c.out32.flatten()])[4:].view_as(c.out32)
    c.run()


@pytest.mark.parametrize("options", [dict(), dict(cap=20.0, spread=3.0, slopes=[0.5]), dict(causal=False), dict(cap=200.0, spread=30.0)])
def test_long_documents_of_few_heads(options):
    """A persistent block takes several items, queries of a key tile are shared, blocks of one query tile."""
    Case([2300], H=1, G=1, seed=22, **options).run()


def test_more_items_than_blocks():
    """Every block takes several items, of one and of two query tiles, with and without keys behind the diagonal."""
    rng = np.random.Generator(np.random.PCG64(7))
    lengths = [int(n) for n in rng.integers(0, 400, 150)]
    for options in (dict(), dict(causal=False), dict(prefix=[int(n) for n in rng.integers(0, 400, 150)], cap=30.0, spread=4.0, slopes=[0.1, 0.5, 1.0, 0.0])):
        Case(lengths, H=4, G=2, d=32, seed=23, **options).run()


def test_halved_blocks_of_one_long_document():
    """All pairs of a document whose last blocks of two query tiles are halved; two rows' results against fp64 by hand."""
    n, H, d = 5000, 16, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(n, H, d, device="cuda", generator=g).bfloat16() for _ in range(3))
    out, lse = torch.full_like(q, LEFT), torch.full((H, n), LEFT, device="cuda")
    gt.gt_check(gt.gt_position_attn_fwd(q, k, v, None, None, gt.Batch(n), False, 0.0, out, lse))
    x = torch.einsum("ihd,jhd->hij", q.double(), k.double()) / d ** 0.5
    ref = torch.einsum("hij,jhd->ihd", torch.softmax(x, 2), v.double())
    assert float((lse.double() - torch.logsumexp(x, 2)).abs().max()) <= 1e-4
    assert float((out.double() - ref).norm() / ref.norm()) <= 2 * ONE


def test_two_calls_at_once_on_two_streams():
    """With workspaces of their own."""
    a, b = Case([700, 100, 300], H=4, G=2, seed=24), Case([512, 33], H=8, G=8, cap=10.0, seed=25)
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    spaces = []
    for _ in range(3):
        for c, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                spaces += [c.forward(), c.backward()]
    torch.cuda.synchronize()
    for ws in spaces:
        gt.gt_check(ws)
    a.check()
    b.check()


def test_counters_are_zero_between_calls():
    """Words of the workspaces' headers that the persistent kernels count with."""
    c = Case([300] * 40, H=8, G=8, d=32, seed=26)
    for ws in (c.forward(), c.backward()):
        torch.cuda.synchronize()
        assert not ws[:256].any()


@pytest.mark.parametrize("options", [dict(), dict(cap=30.0, spread=4.0), dict(causal=False), dict(causal=False, cap=10.0), dict(prefix=[200], cap=50.0)])
def test_slopes_of_either_sign(options):
    """A negative slope is a bonus on distance: the largest scores are the farthest keys'."""
    Case([500], H=4, G=4, slopes=[-0.5, 0.5, -3.0, 0.0], seed=27, **options).run()


@pytest.mark.parametrize("options", [dict(), dict(causal=False), dict(cap=30.0), dict(causal=False, cap=1000.0)])
def test_slopes_that_leave_a_query_itself_only(options):
    """Penalties far beyond the range of the exponentials, up to the largest documented: every query's output is its own value."""
    c = Case([300, 150], H=4, G=4, slopes=[1e3, 1e9, 1e20, 1e27], seed=28, **options)
    gt.gt_check(c.forward())
    gt.gt_check(c.backward())
    ref = c.check(names=("out", "lse", "dv"))
    assert torch.equal(c.out, c.v)
    # dq and dk are 0: what is left of dP - Delta, two sums of the same products in fp32, has the elementwise bound only (a norm that counts
    # roundings of the results to bf16 is 0, too)
    got = c.results()
    for name in ("dq", "dk"):
        assert np.all(np.abs(got[name] - ref[name]) <= ref["bounds"][name]), name


def test_one_row_of_a_projection():
    """A single token's tensors count as packed, whatever stride their only row has."""
    Case([1], H=4, G=2, seed=29, apart=True).run()


@pytest.mark.parametrize("options", [dict(), dict(cap=30.0), dict(slopes=[0.1] * 4)])
def test_terms_beyond_bf16_of_another_document(options):
    """dout . out of a row that shares a tile with the document before it is finite in fp32, but not in bf16."""
    c = Case([100, 28], H=4, G=4, seed=30, **options)
    gt.gt_check(c.forward())
    gt.gt_check(c.backward(exact=False))
    want = [x[:100].clone() for x in (c.dk, c.dv)]
    c.out[100], c.dout[100] = 0.0, 0.0
    c.out[100, :, 0], c.out[100, :, 1] = 1.9921875 * 2.0 ** 64, 0.75 * 2.0 ** 57
    c.dout[100, :, :2] = 2.0 ** 63
    assert bool((c.out[100].float() * c.dout[100].float()).sum(-1).isfinite().all())
    gt.gt_check(c.backward(exact=False))
    assert all(torch.equal(x[:100], y) for x, y in zip((c.dk, c.dv), want))


@pytest.mark.parametrize("options", [dict(), dict(prefix=[9, 200], cap=20.0, slopes=[0.5, 0.0, 0.1, 1.0])])
def test_workspace_at_once_behind_the_results(options):
    """A call without the fp32 output may hand over its workspace where that output would stand."""
    c = Case([100, 300], H=4, G=2, seed=31, **options)
    wf = gt._workspace(gt.gt_position_attn_fwd_workspace(c.batch, 4, 2, 64), "cuda")
    wb = gt._workspace(gt.gt_position_attn_bwd_workspace(c.batch, 4, 2, 64), "cuda")
    assert gt.gt_position_attn_fwd(c.q, c.k, c.v, c.slopes, c.prefix, c.batch, True, c.cap, c.out, c.lse, wf) is wf
    assert gt.gt_position_attn_bwd(c.q, c.k, c.v, c.out, c.dout, c.lse, c.slopes, c.prefix, c.batch, True, c.cap, c.dq, c.dk, c.dv, wb) is wb
    gt.gt_check(wf)
    gt.gt_check(wb)
    c.check(exact=False)
    out32, kept = c.out32.clone(), c.out.clone()
    gt.gt_position_attn_fwd(c.q, c.k, c.v, c.slopes, c.prefix, c.batch, True, c.cap, c.out, c.lse, wf, c.out32)
    gt.gt_check(wf)
    assert not torch.equal(c.out32, out32) and rel_l2(to_f64(c.out), to_f64(kept)) <= 2 * ONE


def _ragged(n, high, seed):
    return [int(x) for x in np.random.Generator(np.random.PCG64(seed)).integers(0, high, n)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("documents", [66, 40])
def test_work_list_with_rows_behind_the_last_document(documents, causal):
    """Ragged documents in the order of the batch and by size, so many that both directions work by a list, and several tiles' rows behind them."""
    Case(_ragged(documents, 900, 32), H=4 if documents > 64 else 8, G=4, d=32, causal=causal, extra=1500, seed=32).run()


def test_work_list_of_a_shorter_batch_in_the_same_workspace_and_graph():
    """The number of rows stays, the documents get shorter from call to call: what an earlier list said must not be read again."""
    lengths = _ragged(66, 900, 33)
    c = Case(lengths, H=4, G=2, d=32, extra=300, seed=33)
    wf, wb = c.forward(), c.backward()
    gt.gt_check(wf)
    gt.gt_check(wb)
    c.check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward(ws=wf)
        c.backward(ws=wb)
    for share in (0.6, 0.1):
        c.cu = np.concatenate([[0], np.cumsum([int(n * share) for n in lengths])]).astype(np.int32)
        c.n = int(c.cu[-1])
        c.batch.cu_seqlens.copy_(torch.from_numpy(c.cu))
        ref = None
        for again in (lambda: (c.forward(ws=wf), c.backward(ws=wb)), g.replay):
            for x in (c.out, c.out32, c.lse, c.dq, c.dk, c.dv):
                x.fill_(LEFT)
            again()
            gt.gt_check(wf)
            gt.gt_check(wb)
            ref = c.check(ref=ref)


def _check_own_sums(c, ref):
    """dq, dk and dv of a backward without the fp32 output: what the roundings of probabilities, dS and results leave."""
    got, n = c.results(), c.n
    for name in ("dq", "dk", "dv"):
        own = name if name == "dv" else name + "_own"
        off = np.abs(got[name][:n] - ref[name])
        assert np.all(off <= ref["bounds"][own]), (name, float((off / ref["bounds"][own]).max()))
        if off.size >= 4096:
            assert np.linalg.norm(off) <= 1.1 * ref["norms"][own], (name, float(np.linalg.norm(off) / ref["norms"][own]))
        assert np.all(got[name][n:] == LEFT), name


@pytest.mark.parametrize("options", [dict(), dict(slopes=[0.5, 0.0625, 0.0, 2.0]), dict(cap=30.0), dict(causal=False), dict(causal=False, cap=5.0, slopes=[0.5, 0.1, 0.0, 1.0]),
                                     dict(prefix=[9, 200, -5, 1 << 30, 3], cap=50.0, slopes=[0.5, 0.0625, 0.0, -0.5]), dict(cap=1e-3), dict(cap=200.0, spread=40.0)])
@pytest.mark.parametrize("lengths", [[600], [16, 16, 0, 300, 33], [1, 2, 128, 129, 257]])
@pytest.mark.parametrize("d", [32, 64])
def test_gradients_without_the_fp32_output(options, lengths, d):
    """Rows of few large probabilities, where dout . out of a bf16 output was off by 0.5 % of dq and more."""
    o = dict(spread=4.0) | options
    if "prefix" in o:
        o["prefix"] = o["prefix"][:len(lengths)]
    c = Case(lengths, H=4, G=2, d=d, seed=34, **o)
    gt.gt_check(c.forward(exact=False))
    gt.gt_check(c.backward(exact=False))
    _check_own_sums(c, c.oracle())


@pytest.mark.parametrize("n", [1, 2, 31, 64, 65, 127, 128, 129, 256, 257, 384, 513])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_without_the_fp32_output(n, causal):
    c = Case([n], H=2, G=1, causal=causal, spread=4.0, seed=n, extra=3, apart=True)
    gt.gt_check(c.forward(exact=False))
    gt.gt_check(c.backward(exact=False))
    _check_own_sums(c, c.oracle())


def test_work_list_without_the_fp32_output():
    for documents, extra in ((66, 700), (30, 0)):
        c = Case(_ragged(documents, 700, 35), H=4, G=4, d=32, spread=4.0, extra=extra, seed=35)
        gt.gt_check(c.forward(exact=False))
        gt.gt_check(c.backward(exact=False))
        _check_own_sums(c, c.oracle())


@pytest.mark.parametrize("options", [dict(), dict(cap=30.0), dict(slopes=[0.1, 0.5, 0.0, 1.0]), dict(causal=False), dict(prefix=[70, 150, 0])])
def test_other_documents_values_do_not_leak_without_the_fp32_output(options):
    kw = dict(lengths=[70, 200, 300], H=4, G=2, extra=40, seed=36, spread=3.0) | options
    clean = Case(**kw)
    clean.forward(exact=False)
    gt.gt_check(clean.backward(exact=False))
    _check_own_sums(clean, clean.oracle())
    for bad in (float("nan"), float("inf")):
        c = Case(**kw)
        for x in (c.q, c.k, c.v, c.dout):
            x[70:270] = bad
            x[570:] = -bad
        gt.gt_check(c.forward(exact=False))
        c.lse[:, 70:270] = bad
        gt.gt_check(c.backward(exact=False))
        for rows in (slice(0, 70), slice(270, 570)):
            assert torch.equal(c.out[rows], clean.out[rows]) and torch.equal(c.lse[:, rows], clean.lse[:, rows])
            for name in ("dq", "dk", "dv"):
                x, y = to_f64(getattr(c, name)[rows]), to_f64(getattr(clean, name)[rows])
                assert np.isfinite(x).all() and rel_l2(x, y) <= 2 * ONE, name              # (the order of the sums)


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("options", [dict(), dict(cap=30.0), dict(slopes=[0.1] * 4)])
def test_terms_beyond_bf16_leave_the_rest_of_their_own_document(options, exact):
    """dout . out of one query overflows: dv does not depend on it, nor do the gradients of queries and heads beside it."""
    c = Case([100, 28], H=4, G=4, seed=37, **options)
    gt.gt_check(c.forward())
    row, big = 110, 2.0 ** 63
    c.dout[row, 1, :2] = big
    if exact:
        c.out32[row, 1, :2] = 2.0 ** 66
    else:                                                # (the backward's own Delta: sums of dout . v)
        c.v[100:row + 1, 1, :2] = 2.0 ** 66
        gt.gt_check(c.forward())
    gt.gt_check(c.backward(exact))
    ref, got = c.oracle(), c.results()
    assert np.all(np.abs(got["dv"] - ref["dv"]) <= ref["bounds"]["dv"])
    others = [h for h in range(4) if h != 1]
    for name in ("dq", "dk"):
        limit = ref["bounds"][name if exact else name + "_own"]
        assert np.all(np.abs(got[name] - ref[name])[:, others] <= limit[:, others]), name
        assert np.all(np.abs(got[name] - ref[name])[:100] <= limit[:100]), name
    assert np.all(np.abs(got["dq"] - ref["dq"])[row + 1:] <= ref["bounds"]["dq" if exact else "dq_own"][row + 1:])


@pytest.mark.parametrize("options", [dict(cap=30.0), dict(cap=200.0), dict(slopes=[0.5, 0.1, 0.0, -0.5]), dict(prefix=[70, 150, 100]), dict(causal=False, cap=10.0),
                                     dict(causal=False, slopes=[0.5, 0.1, 0.0, 1.0]), dict(prefix=[3, 300, 299], cap=50.0, slopes=[0.5, 0.1, 0.0, 1.0])])
@pytest.mark.parametrize("d", [32, 64])
def test_other_documents_values_do_not_leak_with_options(options, d):
    """As above, with caps (one that bounds the scores, one that does not), penalties and prefixes, in a batch that works by the list, too."""
    kw = dict(lengths=[70, 200, 300], H=4, G=2, d=d, extra=40, seed=38, spread=2.0) | options
    clean = Case(**kw)
    clean.run()
    for bad in (float("nan"), float("inf")):
        c = Case(**kw)
        for x in (c.q, c.k, c.v, c.dout):
            x[70:270] = bad
            x[570:] = -bad
        gt.gt_check(c.forward())
        c.lse[:, 70:270] = bad
        c.out32[70:270] = bad
        gt.gt_check(c.backward())
        for rows in (slice(0, 70), slice(270, 570)):
            assert torch.equal(c.out[rows], clean.out[rows]) and torch.equal(c.lse[:, rows], clean.lse[:, rows])
            for name in ("dq", "dk", "dv"):
                x, y = to_f64(getattr(c, name)[rows]), to_f64(getattr(clean, name)[rows])
                assert np.isfinite(x).all() and rel_l2(x, y) <= 2 * ONE, name              # (the order of the sums)
        assert bool((c.out[570:] == LEFT).all()) and bool((c.dk[570:] == LEFT).all())


@pytest.mark.parametrize("exact", [True, False])
@pytest.mark.parametrize("prefix", [1, 129, 700, 1500, 2300])
def test_shared_key_tiles_with_a_prefix_and_rows_apart(prefix, exact):
    """One head of a long document: several items share a key tile's queries, from the prefix's beginning or from the tile on."""
    c = Case([2300], H=1, G=1, prefix=[prefix], extra=60, seed=39, apart=True, spread=2.0)
    gt.gt_check(c.forward(exact))
    gt.gt_check(c.backward(exact))
    c.check(exact)
    if not exact:
        _check_own_sums(c, c.oracle())


def test_shared_key_tiles_of_several_documents_with_options():
    Case([1300, 0, 900], H=2, G=1, prefix=[400, 5, 900], slopes=[0.1, 0.5], cap=20.0, extra=200, seed=40, apart=True, spread=3.0).run()


def test_captured_and_on_two_streams_without_the_fp32_output():
    """The pass for Delta in a graph that is replayed on other inputs, and twice at once with workspaces of their own."""
    c = Case(_ragged(40, 400, 41), H=8, G=8, d=32, spread=4.0, extra=200, seed=41)
    wf, wb = c.forward(exact=False), c.backward(exact=False)
    gt.gt_check(wb)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.forward(exact=False, ws=wf)
        c.backward(exact=False, ws=wb)
    other = Case(_ragged(40, 400, 41), H=8, G=8, d=32, spread=4.0, extra=200, seed=42)
    for x in ("q", "k", "v", "dout"):
        getattr(c, x).copy_(getattr(other, x))
    for x in (c.out, c.lse, c.dq, c.dk, c.dv):
        x.fill_(LEFT)
    g.replay()
    gt.gt_check(wf)
    gt.gt_check(wb)
    _check_own_sums(c, c.oracle())
    a, b = Case([700, 100, 300], H=4, G=2, spread=4.0, seed=43), Case([512, 33], H=8, G=8, cap=10.0, spread=3.0, seed=44)
    torch.cuda.synchronize()
    streams, spaces = (torch.cuda.Stream(), torch.cuda.Stream()), []
    for _ in range(3):
        for x, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                spaces += [x.forward(exact=False), x.backward(exact=False)]
    torch.cuda.synchronize()
    for ws in spaces:
        gt.gt_check(ws)
    for x in (a, b):
        _check_own_sums(x, x.oracle())


@pytest.mark.parametrize("options", [dict(), dict(causal=False), dict(cap=30.0), dict(causal=False, cap=1000.0)])
def test_slopes_that_leave_a_query_itself_only_without_the_fp32_output(options):
    """Delta is then dP itself, to the rounding of a quotient: what is left of their difference has the elementwise bound."""
    c = Case([300, 150], H=4, G=4, slopes=[1e3, 1e9, 1e20, 1e27], seed=45, **options)
    gt.gt_check(c.forward(exact=False))
    gt.gt_check(c.backward(exact=False))
    ref, got = c.check(exact=False, names=("out", "lse", "dv")), c.results()
    for name in ("dq", "dk"):
        assert np.all(np.abs(got[name] - ref[name]) <= ref["bounds"][name + "_own"]), name


@pytest.mark.parametrize("options", [dict(), dict(cap=30.0, spread=4.0), dict(causal=False), dict(causal=False, cap=10.0), dict(prefix=[200], cap=50.0)])
def test_slopes_of_either_sign_without_the_fp32_output(options):
    c = Case([500], H=4, G=4, slopes=[-0.5, 0.5, -3.0, 0.0], seed=46, **options)
    gt.gt_check(c.forward(exact=False))
    gt.gt_check(c.backward(exact=False))
    _check_own_sums(c, c.oracle())
