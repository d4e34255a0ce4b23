"""GPU parity of the context-cache operators against oracle/cache.py.

Tolerances.  Attention outputs and log-sum-exps: those of gpu_helpers.TOL, which
hold for any set of visible keys.  4-bit codes, scale bytes, copies and
evictions: exact.  Weights: see _weight_bound.
"""

import numpy as np
import pytest
import torch

import paper_2609_00355_amd as G
from oracle import cache as OC
from workloads import trees as WT

from gpu_helpers import assert_close, ensure_lib

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    ensure_lib()


def _np(t):
    return t.detach().float().cpu().numpy() if t.dtype == torch.bfloat16 else t.detach().cpu().numpy()


class Case:
    """Inputs of one call: on the host as float64 (what the tensors hold) and on the GPU."""

    def __init__(self, dtype, fmt, d, n, hq, hkv, lens, cap=None, seed=0, sharp=1.0, poison=False, n_sinks=0, window=0, weights=False):
        g = torch.Generator().manual_seed(seed)
        dt = DT[dtype]
        b = len(lens)
        cap = max(max(lens), 1) if cap is None else cap

        def normal(*shape):
            return torch.randn(*shape, generator=g)

        self.dtype, self.fmt, self.n, self.lens = dtype, fmt, n, np.array(lens, dtype=np.int32)
        self.q, self.k_new, self.v_new = (x.to(dt) for x in (normal(b, n, hq, d) * sharp, normal(b, n, hkv, d), normal(b, n, hkv, d)))
        self.parents = torch.tensor(np.stack([WT.best_first_tree(n, 15, (1, 2, 4), 1000, (seed, i))[0] for i in range(b)]))
        k, v = normal(b, hkv, cap, d).to(dt), normal(b, hkv, cap, d).to(dt)
        hidden = np.ones((b, cap), dtype=bool)  # slots that no row sees
        for i, ctx in enumerate(lens):
            hidden[i, :ctx] = False
            if window:
                hidden[i, min(n_sinks, ctx):max(min(n_sinks, ctx), min(ctx, ctx - window + 1))] = True
        hidden = torch.tensor(hidden)[:, None, :, None]
        if fmt == "kv4":
            (ck, sk), (cv, sv) = OC.encode(k.float()), OC.encode(v.float())
            if poison:
                hid = hidden.numpy()
                sk, sv = np.where(hid, np.uint8(255), sk), np.where(hid, np.uint8(255), sv)
            pk, pv = OC.pack(ck), OC.pack(cv)
            self.k64, self.v64 = OC.decode(pk, sk), OC.decode(pv, sv)
            dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (pk, pv, sk, sv)]
            self.cache = G.ContextCache(dev[0], dev[1], None, k_scale=dev[2], v_scale=dev[3])
        else:
            if poison:
                k, v = k.masked_fill(hidden, float("nan")), v.masked_fill(hidden, float("nan"))
            self.k64, self.v64 = k.double().numpy(), v.double().numpy()
            self.cache = G.ContextCache(k.cuda(), v.cuda(), None)
        self.cache.ctx_lens = torch.tensor(self.lens).cuda()
        self.weights = None
        if weights:
            self.weights = torch.rand(b, hkv, cap, generator=g)
            self.cache.weights = self.weights.cuda()

    def attn(self, tree, n_sinks=0, window=0, **kw):
        q, kn, vn = self.q.cuda(), self.k_new.cuda(), self.v_new.cuda()
        if tree:
            return G.glance_cache_tree_verify_attn(q, self.cache, kn, vn, self.parents.cuda(), n_sinks, window, **kw)
        return G.glance_cache_block_draft_attn(q, self.cache, kn, vn, n_sinks, window, **kw)

    def want(self, tree, n_sinks=0, window=0):
        return OC.attention(self.q.double(), self.k64, self.v64, self.k_new.double(), self.v_new.double(), self.lens,
                            self.parents.numpy() if tree else None, n_sinks, window)

    def check(self, tree, n_sinks=0, window=0):
        out, lse = self.attn(tree, n_sinks, window)
        torch.cuda.synchronize()
        ref = self.want(tree, n_sinks, window)
        assert_close(_np(out), _np(lse), *ref, self.dtype, f"{self.fmt} {self.dtype} sinks {n_sinks} window {window}")
        return out, lse


# ------------------------------------------------------------- attention
REACH = [(0, 1), (0, 2), (3, 1), (0, 17), (5, 64), (64, 65), (70, 100), (0, 129), (1, 300), (1000, 5), (200, 260), (0, 10 ** 6), (0, 0)]


@pytest.mark.parametrize("n_sinks,window", REACH)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_reach(fmt, dtype, tree, n_sinks, window):
    """Windows and sinks around the tile sizes over lengths around them; what no row sees is NaN."""
    c = Case(dtype, fmt, 64, 9, 4, 2, [0, 1, 15, 16, 17, 63, 64, 65, 128, 200, 321], cap=330, seed=window, poison=True, n_sinks=n_sinks,
             window=window)
    c.check(tree, n_sinks, window)


@pytest.mark.parametrize("n,hq,hkv", [(1, 4, 4), (1, 28, 4), (2, 16, 1), (64, 14, 2), (33, 6, 3), (64, 16, 1), (16, 28, 4)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_head_layouts(fmt, dtype, d, n, hq, hkv):
    lens = [513, 40] if dtype == "f32" else [700, 5, 333]
    c = Case(dtype, fmt, d, n, hq, hkv, lens, seed=n + d, poison=True, n_sinks=4, window=150)
    c.check(True, 4, 150)
    c = Case(dtype, fmt, d, n, hq, hkv, lens, seed=n + d + 1, poison=True)
    c.check(False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_long_contexts_in_many_pieces(fmt, dtype):
    c = Case(dtype, fmt, 128, 7, 4, 1, [5003, 0, 1999], seed=5, sharp=3.0, poison=True, n_sinks=100, window=3000)
    c.check(True, 100, 3000)
    c = Case(dtype, fmt, 64, 3, 2, 1, [7001], seed=6, sharp=3.0)
    c.check(False)


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_more_sequences_than_lanes(fmt):
    lens = [(37 * i) % 150 for i in range(70)]
    c = Case("bf16", fmt, 64, 2, 2, 2, lens, seed=9, poison=True, n_sinks=2, window=40)
    c.check(True, 2, 40)
    c.check(False, 2, 40)


def test_window_shorter_than_the_tree():
    """A chain of 64: deep nodes see only the nearest ancestors and the sinks among them."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, "dense", 64, 64, 2, 1, [2, 0, 90], seed=11)
        c.parents = torch.arange(-1, 63, dtype=torch.int32).repeat(3, 1)
        for n_sinks, window in ((0, 1), (4, 3), (10, 20), (100, 1)):
            c.check(True, n_sinks, window)


def test_whole_dense_cache_agrees_with_the_plain_call():
    """Without a window both entry points compute the same attention."""
    c = Case("f32", "dense", 128, 16, 8, 2, [300, 77], seed=12)
    a = c.attn(True)
    b = G.glance_tree_verify_attn(c.q.cuda(), c.cache.k, c.cache.v, c.k_new.cuda(), c.v_new.cuda(), c.cache.ctx_lens, c.parents.cuda())
    torch.testing.assert_close(a[0], b[0], rtol=0, atol=1e-5)
    torch.testing.assert_close(a[1], b[1], rtol=0, atol=1e-5)


def test_lengths_out_of_range_are_clamped():
    c = Case("bf16", "kv4", 64, 4, 2, 2, [120, 0, 64], cap=120, seed=13)
    want = c.attn(True, 3, 50)
    c.cache.ctx_lens = torch.tensor([10 ** 9, -5, 64], dtype=torch.int32).cuda()
    got = c.attn(True, 3, 50)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_empty_cache():
    for dtype in ("bf16", "f32"):
        for fmt in ("dense", "kv4"):
            c = Case(dtype, fmt, 64, 5, 4, 2, [0, 0], cap=1, seed=14, poison=True)
            c.check(True, 2, 3)
        e = G.new_cache(2, 2, 0, 64, dtype=DT[dtype])
        c.cache, c.k64, c.v64 = e, np.zeros((2, 2, 0, 64)), np.zeros((2, 2, 0, 64))
        c.fmt = "dense"
        c.check(False)


# ------------------------------------------------------------- 4-bit caches
def _hard_values(rows, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, d, generator=g) * torch.exp(4 * torch.randn(rows, 1, generator=g))
    grid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 6.9, 0.0, -0.0, 3.0, 0.24, 0.26, 5.01])
    x[0, :16], x[0, 16:32] = grid, -grid
    x[1] = 0.0
    x[2, 3] = 7.0
    x[3] = 2.0 ** -140 if dtype == "f32" else 2.0 ** -130
    x[4, :] = 3.0e38
    x[5, 40], x[6, 1], x[7, 33] = float("nan"), float("inf"), float("-inf")
    return x.to(DT[dtype])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_convert(dtype, d):
    """Codes, scales and values, bit for bit; slots past the lengths are left alone."""
    b, hkv, cap = 3, 2, 70
    lens = np.array([70, 0, 33], dtype=np.int32)
    k = _hard_values(b * hkv * cap, d, dtype, 1).reshape(b, hkv, cap, d)
    v = _hard_values(b * hkv * cap, d, dtype, 2).reshape(b, hkv, cap, d)
    src = G.ContextCache(k.cuda(), v.cuda(), torch.tensor(lens).cuda())
    dst = G.new_cache(b, hkv, 50, d, fmt="kv4")  # smaller: cut there
    for t in (dst.k, dst.v, dst.k_scale, dst.v_scale):
        t.fill_(0x5a)
    G.glance_cache_convert(src, dst)
    want_len = np.minimum(lens, 50)
    assert dst.ctx_lens.cpu().tolist() == want_len.tolist()
    back = G.new_cache(b, hkv, 64, d, dtype=DT[dtype])
    back.k.fill_(9.0)
    G.glance_cache_convert(dst, back)
    torch.cuda.synchronize()
    assert back.ctx_lens.cpu().tolist() == want_len.tolist()
    for x, p, s, r in ((k, dst.k, dst.k_scale, back.k), (v, dst.v, dst.v_scale, back.v)):
        codes, scales = OC.encode(x.float()[:, :, :50])
        nan = np.repeat(scales == 255, 16, axis=-1)
        for i, n in enumerate(want_len):
            assert np.array_equal(s.cpu().numpy()[i, :, :n], scales[i, :, :n])
            got, ref = p.cpu().numpy()[i, :, :n], OC.pack(codes)[i, :, :n]
            assert np.array_equal(np.where(nan[i, :, :n], 0, got), np.where(nan[i, :, :n], 0, ref))
            assert (p.cpu().numpy()[i, :, n:] == 0x5a).all() and (s.cpu().numpy()[i, :, n:] == 0x5a).all()
            np.testing.assert_array_equal(_np(r)[i, :, :n], OC.decode(ref, scales[i, :, :n]).astype(np.float32))
    assert (_np(back.k)[1] == 9.0).all()


def test_values_that_read_nan_reach_the_output():
    """A block with a NaN makes the rows that see it NaN, and no other sequence's."""
    c = Case("bf16", "kv4", 64, 2, 2, 1, [100, 100], seed=3)
    c.cache.k_scale[0, 0, 10, 0] = 255
    out, _ = c.attn(False)
    assert torch.isnan(out[0]).all() and torch.isfinite(out[1]).all()
    out, _ = c.attn(False, 0, 50)  # outside the window it is not read
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_commit(fmt, dtype, d):
    b, n, hkv, cap = 4, 20, 3, 48
    c = Case(dtype, fmt, d, n, hkv, hkv, [0, 20, 45, 48], cap=cap, seed=d)
    alen = np.array([5, 2, 6, 1], dtype=np.int32)
    path = np.full((b, 8), -1, dtype=np.int32)
    for i, a in enumerate(alen):
        path[i, :a + 1] = np.sort(np.random.default_rng(i).choice(n, a + 1, replace=False))
    path[1, 2] = 77  # not a node: the copy ends there
    before = [t.clone() for t in (c.cache.k, c.cache.v)]
    G.glance_cache_commit_path(c.cache, c.k_new.cuda(), c.v_new.cuda(), torch.tensor(alen).cuda(), torch.tensor(path).cuda())
    torch.cuda.synchronize()
    lens = [0 + 6, 20 + 2, 48, 48]
    assert c.cache.ctx_lens.cpu().tolist() == lens
    for new, t, s, old in ((c.k_new, c.cache.k, c.cache.k_scale, before[0]), (c.v_new, c.cache.v, c.cache.v_scale, before[1])):
        for i in range(b):
            start = int(c.lens[i])
            for t_, slot in enumerate(range(start, lens[i])):
                row = new[i, path[i, t_]]
                if fmt == "dense":
                    assert torch.equal(t[i, :, slot].cpu(), row)
                else:
                    codes, scales = OC.encode(row.float())
                    assert np.array_equal(t[i, :, slot].cpu().numpy(), OC.pack(codes))
                    assert np.array_equal(s[i, :, slot].cpu().numpy(), scales)
            assert torch.equal(t[i, :, :start], old[i, :, :start]) and torch.equal(t[i, :, lens[i]:], old[i, :, lens[i]:])


# ------------------------------------------------------------- weights
def _weight_bound(c, lse, rows_per_head, ref):
    """Derived: a weight is a sum of exp2 of scale * s - lse in fp32.  The products are exact (bf16) or
    rounded once, and D terms are summed, so the score is off by at most (D + 1) 2^-24 sum |q k|; the
    argument's multiply-add and lse's scaling add 2^-23 of the largest argument, exp2 an ulp, and the sum
    over R rows R 2^-24 relative.  All of it is relative to the weight."""
    d = c.q.shape[-1]
    reach = c.q.double().abs().max(0).values.max(0).values.max(0).values.numpy()  # largest |q| of each dim
    keys = max((np.abs(x).reshape(-1, d) @ reach).max() for x in (c.k64, c.k_new.double().numpy()))  # sum |q k|
    arg = keys / np.sqrt(d) + np.abs(lse).max()
    rel = 2.0 ** -24 * ((d + 1) * keys / np.sqrt(d) + 3 * 1.4427 * arg + 4 + rows_per_head)
    return rel * np.abs(ref) + 1e-30


@pytest.mark.parametrize("n_sinks,window", [(0, 0), (5, 40), (0, 1), (70, 3), (0, 200)])
@pytest.mark.parametrize("path", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["dense", "kv4"])
@pytest.mark.parametrize("d,n,hq,hkv", [(64, 20, 4, 2), (128, 64, 14, 2), (128, 1, 16, 1)])
def test_weigh(fmt, dtype, d, n, hq, hkv, path, n_sinks, window):
    lens = [0, 1, 64, 65, 130, 300]
    c = Case(dtype, fmt, d, n, hq, hkv, lens, cap=304, seed=window + n, poison=False, weights=True)
    rng = np.random.default_rng(n + window)
    lse = c.want(True, n_sinks, window)[1] if path else c.want(False, n_sinks, window)[1]
    lse = torch.tensor(lse, dtype=torch.float32)
    kw = {}
    if path:
        alen = np.zeros(len(lens), dtype=np.int32)
        nodes = np.full((len(lens), 16), -1, dtype=np.int32)
        for b in range(len(lens)):
            v, chain = int(rng.integers(n)), []
            while v >= 0:
                chain.append(v)
                v = int(c.parents[b, v])
            alen[b] = len(chain) - 1
            nodes[b, :len(chain)] = chain[::-1]
        alen[2] = -1  # nothing accepted, not even the root
        kw = dict(k_new=c.k_new, accept_len=torch.tensor(alen), accept_path=torch.tensor(nodes))
    for decay in (1.0, 0.5, 0.0):
        dev = {k: v.cuda() for k, v in kw.items()}
        into = torch.full_like(c.cache.weights, 7.0)
        got = G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=decay, n_sinks=n_sinks, window=window, weights_out=into, **dev)
        torch.cuda.synchronize()
        assert torch.equal(c.cache.weights.cpu(), c.weights)  # an output of its own leaves the cache's alone
        ref = OC.weigh(c.q.double(), c.k64, lse.double(), c.lens, c.weights.double(), decay, n_sinks=n_sinks, window=window,
                       **{k: (v.double().numpy() if k == "k_new" else v.numpy()) for k, v in kw.items()})
        got = got.cpu().numpy()
        for b, ctx in enumerate(lens):
            end = ctx + (min(len(OC.path_nodes(alen[b], nodes[b], n)), 304 - ctx) if path else 0)
            bound = _weight_bound(c, lse.numpy(), n * hq // hkv, ref[b, :, :end])
            assert (np.abs(got[b, :, :end] - ref[b, :, :end]) <= bound).all(), (b, decay, np.abs(got[b, :, :end] - ref[b, :, :end]).max())
            assert (got[b, :, end:] == 7.0).all()
    # in place, with NaN in the old weights and decay 0
    c.cache.weights.fill_(float("nan"))
    dev = {k: v.cuda() for k, v in kw.items()}
    G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=0.0, n_sinks=n_sinks, window=window, **dev)
    assert torch.isfinite(c.cache.weights[5, :, :300]).all()
    if not path:
        assert torch.equal(c.cache.weights[5, :, :300].cpu(), torch.tensor(got[5, :, :300]))


@pytest.mark.parametrize("lens", [[60, 50], [120, 90], [200, 190], [330, 100], [600, 610], [1500, 901]])
@pytest.mark.parametrize("fmt,dtype", [("dense", "bf16"), ("kv4", "bf16"), ("dense", "f32"), ("kv4", "f32")])
def test_weigh_in_pieces_of_every_length(fmt, dtype, lens):
    """Many KV heads, so few workgroups a head: from one step to more steps than waves each."""
    hkv, n = 64, 40
    c = Case(dtype, fmt, 64, n, hkv, hkv, lens, seed=lens[0], weights=True)
    for window, n_sinks in ((0, 0), (70, 3)):
        lse = torch.tensor(c.want(False, n_sinks, window)[1], dtype=torch.float32)
        into = torch.zeros_like(c.cache.weights)
        got = G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=0.5, n_sinks=n_sinks, window=window, weights_out=into).cpu().numpy()
        ref = OC.weigh(c.q.double(), c.k64, lse.double(), c.lens, c.weights.double(), 0.5, n_sinks=n_sinks, window=window)
        for b, ctx in enumerate(lens):
            bound = _weight_bound(c, lse.numpy(), n, ref[b, :, :ctx])
            assert (np.abs(got[b, :, :ctx] - ref[b, :, :ctx]) <= bound).all(), (b, window)
            assert (got[b, :, ctx:] == 0).all()


# ------------------------------------------------------------- eviction
@pytest.mark.parametrize("fmt,dtype,d", [("dense", "bf16", 128), ("dense", "f32", 64), ("kv4", "bf16", 64), ("kv4", "bf16", 128)])
@pytest.mark.parametrize("budget,n_sinks,n_recent", [(1, 0, 0), (1, 1, 0), (2, 1, 1), (63, 0, 63), (64, 4, 16), (100, 0, 0), (600, 17, 33),
                                                     (1025, 0, 1), (3000, 1, 2)])
def test_evict(fmt, dtype, d, budget, n_sinks, n_recent):
    lens = [0, 1, 64, 1024, 1025, 2700, budget]
    c = Case(dtype, fmt, d, 1, 2, 2, lens, cap=max(lens) + 3, seed=budget, weights=True)
    rng = np.random.default_rng(budget)
    w = np.exp(3 * rng.normal(size=tuple(c.weights.shape))).astype(np.float32)
    w[rng.random(w.shape) < 0.3] = 0.0      # many ties
    w[0], w[5, 0] = -w[0], 0.25             # one head all equal
    w[4, 0, ::7] = np.nan
    w[3, 0, ::5], w[3, 0, 1::5], w[3, 1, ::9] = -0.0, -2.5, np.inf
    c.cache.weights = torch.tensor(w).cuda()
    to = G.new_cache(len(lens), 2, budget + 2, d, dtype=DT[dtype], fmt=fmt, weights=True)
    fill = [t for t in (to.k, to.v, to.k_scale, to.v_scale, to.weights) if t is not None]
    for t in fill:
        t.fill_(7)
    kept = G.glance_cache_evict(c.cache, to, budget, n_sinks, n_recent)
    torch.cuda.synchronize()
    want = OC.evict(lens, w, budget, n_sinks, n_recent)
    assert to.ctx_lens.cpu().tolist() == [min(x, budget) for x in lens]
    pairs = [(t, s) for t, s in ((to.k, c.cache.k), (to.v, c.cache.v), (to.k_scale, c.cache.k_scale), (to.v_scale, c.cache.v_scale),
                                 (to.weights[..., None], c.cache.weights[..., None])) if t is not None]
    for b in range(len(lens)):
        for g in range(2):
            slots = want[b][g]
            assert kept[b, g].cpu().tolist() == slots + [-1] * (budget - len(slots))
            for t, s in pairs:
                a, r = t[b, g, :len(slots)].cpu(), s[b, g].cpu()[slots]
                assert torch.equal(a.view(torch.uint8), r.contiguous().view(torch.uint8))
                assert (t[b, g, len(slots):] == 7).all()


def test_evict_from_long_contexts():
    """More slots than the selection holds at a time, few and many equal weights, more kept slots than it stages."""
    lens, budget = [70001, 32769, 33000], 9000
    g = torch.Generator().manual_seed(2)
    w = torch.rand(3, 1, 70001, generator=g)
    w[1] = (w[1] * 4).floor() / 4       # four values: thousands of ties
    w[2, 0, ::2] = 0.5
    k = torch.arange(70001, dtype=torch.float32).reshape(1, 1, -1, 1).expand(3, 1, -1, 64).contiguous().cuda()
    src = G.ContextCache(k, k.clone(), torch.tensor(lens, dtype=torch.int32).cuda(), weights=w.cuda())
    to = G.new_cache(3, 1, budget, 64, dtype=torch.float32, weights=True)
    kept = G.glance_cache_evict(src, to, budget, 10, 700)
    torch.cuda.synchronize()
    want = OC.evict(lens, w.numpy(), budget, 10, 700)
    for b in range(3):
        assert kept[b, 0].cpu().tolist() == want[b][0]
        assert to.v[b, 0, :, 63].cpu().tolist() == [float(x) for x in want[b][0]]


def test_evict_with_every_key_held():
    """The longest caches whose keys the selection holds: few heads with many workgroups each, and shares that end inside a chunk."""
    lens, cap = [32768, 30000, 17], 32768
    g = torch.Generator().manual_seed(4)
    w = torch.rand(3, 2, cap, generator=g)
    w[1] = (w[1] * 4).floor() / 4
    k = torch.arange(cap, dtype=torch.float32).reshape(1, 1, -1, 1).expand(3, 2, -1, 64).contiguous().cuda()
    src = G.ContextCache(k, k + 0.5, torch.tensor(lens, dtype=torch.int32).cuda(), weights=w.cuda())
    for budget, n_sinks, n_recent in ((9001, 10, 700), (32767, 0, 0), (3, 1, 1), (5000, 2000, 3000)):
        to = G.new_cache(3, 2, budget, 64, dtype=torch.float32, weights=True)
        kept = G.glance_cache_evict(src, to, budget, n_sinks, n_recent)
        torch.cuda.synchronize()
        want = OC.evict(lens, w.numpy(), budget, n_sinks, n_recent)
        assert to.ctx_lens.cpu().tolist() == [min(x, budget) for x in lens]
        for b in range(3):
            for h in range(2):
                slots = want[b][h]
                assert kept[b, h].cpu().tolist() == slots + [-1] * (budget - len(slots))
                assert to.k[b, h, :len(slots), 0].cpu().tolist() == [float(x) for x in slots]
                assert to.v[b, h, :len(slots), 63].cpu().tolist() == [x + 0.5 for x in slots]
                assert torch.equal(to.weights[b, h, :len(slots)].cpu(), w[b, h][slots])
                assert (to.k[b, h, len(slots):] == 0).all()


@pytest.mark.parametrize("close", [100, 1000, 3000, 5000])
def test_evict_among_close_weights(close):
    """Weights a few units of the last place apart, within a wide range of others: every level of the selection counts."""
    cap = 6000
    rng = np.random.default_rng(close)
    w = np.exp(3 * rng.normal(size=(2, 2, cap))).astype(np.float32) * 1e-3
    w[:, :, :50] = 0.0
    for h in range(4):
        ulps = 37 * np.arange(close) + rng.integers(0, 3, size=close)
        at = rng.permutation(cap)[:close]
        w.reshape(4, cap)[h, at] = (np.float32(1.0).view(np.int32) + ulps.astype(np.int32)).view(np.float32)
    k = torch.arange(cap, dtype=torch.float32).reshape(1, 1, -1, 1).expand(2, 2, -1, 64).contiguous().cuda()
    src = G.ContextCache(k, k.clone(), torch.tensor([cap, cap - 7], dtype=torch.int32).cuda(), weights=torch.tensor(w).cuda())
    for budget in (1, close // 3, close // 2 + 41, close, 2500):
        to = G.new_cache(2, 2, budget, 64, dtype=torch.float32, weights=True)
        kept = G.glance_cache_evict(src, to, budget, 0, 0)
        want = OC.evict([cap, cap - 7], w, budget, 0, 0)
        for b in range(2):
            for h in range(2):
                assert kept[b, h].cpu().tolist() == want[b][h], (budget, b, h)
                assert to.v[b, h, :, 5].cpu().tolist() == [float(x) for x in want[b][h]]


def test_evict_with_shared_lengths():
    c = Case("bf16", "dense", 64, 1, 2, 2, [200, 30], seed=1, weights=True)
    to = G.new_cache(2, 2, 64, 64, weights=True)
    to.ctx_lens = c.cache.ctx_lens
    kept = G.glance_cache_evict(c.cache, to, 64, 1, 2)
    torch.cuda.synchronize()
    assert to.ctx_lens.cpu().tolist() == [64, 30]
    want = OC.evict([200, 30], c.weights.numpy(), 64, 1, 2)
    assert kept[0, 1].cpu().tolist() == want[0][1] and kept[1, 0, :30].cpu().tolist() == list(range(30))


# ------------------------------------------------------------- long caches
@pytest.mark.parametrize("fmt,dtype,d,hkv,cap", [("dense", "bf16", 128, 2, 2 ** 24 + 3), ("dense", "f32", 64, 2, 2 ** 24 + 3),
                                                 ("kv4", "bf16", 128, 4, 2 ** 25), ("kv4", "f32", 128, 4, 2 ** 25)])
def test_offsets_past_32_bits(fmt, dtype, d, hkv, cap):
    """The last slots of a cache of more than 8 GB: what a window and the sinks see there equals a short cache of those slots."""
    sinks, window, n, last = 3, 500, 20, 600
    c = Case(dtype, fmt, d, n, 2 * hkv, hkv, [sinks + last], seed=cap % 97, weights=True)
    ctx = cap - 8
    big = G.new_cache(1, hkv, cap, d, dtype=DT[dtype], fmt=fmt, weights=True)
    for t, s in ((big.k, c.cache.k), (big.v, c.cache.v), (big.k_scale, c.cache.k_scale), (big.v_scale, c.cache.v_scale)):
        if t is not None:
            t[:, :, :sinks], t[:, :, ctx - last:ctx] = s[:, :, :sinks], s[:, :, sinks:]
    big.ctx_lens.fill_(ctx)
    big.weights.fill_(1.0)
    c.cache = big
    out, lse = c.check(True, sinks, window)
    block = c.check(False, sinks, window)[1]
    G.glance_cache_weigh(c.q.cuda(), big, block, decay=0.5, n_sinks=sinks, window=window)
    torch.cuda.synchronize()
    ref = OC.weigh(c.q.double(), c.k64, block.double().cpu(), c.lens, np.ones((1, hkv, sinks + last)), 0.5, n_sinks=sinks, window=window)
    got = _np(torch.cat([big.weights[:, :, :sinks], big.weights[:, :, ctx - last:ctx]], dim=2))
    assert (np.abs(got - ref) <= _weight_bound(c, _np(block), 2 * n, ref)).all()
    assert (big.weights[:, :, sinks:ctx - last] == 0.5).all() and (big.weights[:, :, ctx:] == 1.0).all()

    # committed at the end, and kept by an eviction whose weights name 300 slots
    path = torch.tensor([[0, 5, 6]], dtype=torch.int32).cuda()
    G.glance_cache_commit_path(big, c.k_new.cuda(), c.v_new.cuda(), torch.tensor([2], dtype=torch.int32).cuda(), path)
    assert big.ctx_lens.item() == ctx + 3
    rng = np.random.default_rng(0)
    slots = np.sort(rng.choice(np.arange(10, ctx - 20), size=(hkv, 300)), axis=1)
    big.weights.zero_()
    want = []
    for g in range(hkv):
        mine = np.unique(slots[g])
        big.weights[0, g, torch.tensor(mine).cuda()] = torch.rand(len(mine)).cuda() + 1
        want.append(list(range(8)) + mine.tolist() + list(range(ctx + 3 - 12, ctx + 3)))
    budget = min(len(x) for x in want)
    want = [x if len(x) == budget else None for x in want]
    to = G.new_cache(1, hkv, budget, d, dtype=DT[dtype], fmt=fmt, weights=True)
    kept = G.glance_cache_evict(big, to, budget, 8, 12)
    torch.cuda.synchronize()
    for g in range(hkv):
        if want[g] is not None:
            assert kept[0, g].cpu().tolist() == want[g]
        for t, s in ((to.k, big.k), (to.v, big.v), (to.k_scale, big.k_scale), (to.v_scale, big.v_scale)):
            if t is not None:
                assert torch.equal(t[0, g], torch.stack([s[0, g, j] for j in kept[0, g].tolist()]))
    if fmt == "dense":
        assert torch.equal(to.k[0, :, -3:].cpu(), c.k_new[0, [0, 5, 6]].transpose(0, 1))


# ------------------------------------------------------------- together
def _rounds(fmt, dtype, stream=None, rounds=4):
    """Verify, accept, weigh, commit and (when the cache is full) evict, as a serving loop does; every step against the oracle."""
    b, n, hq, hkv, d, vocab, cap, budget, sinks, recent, window = 2, 24, 4, 2, 64, 50, 96, 64, 4, 16, 80
    g = torch.Generator().manual_seed(3)
    dt = DT[dtype]

    def normal(*shape):
        return torch.randn(*shape, generator=g)

    prefill = G.ContextCache(normal(b, hkv, cap, d).to(dt).cuda(), normal(b, hkv, cap, d).to(dt).cuda(),
                             torch.tensor([70, 41], dtype=torch.int32).cuda())
    caches = [G.new_cache(b, hkv, cap, d, dtype=dt, fmt=fmt, weights=True) for _ in range(2)]
    if fmt == "kv4":
        G.glance_cache_convert(prefill, caches[0])
    else:
        for name in ("k", "v", "ctx_lens"):
            getattr(caches[0], name).copy_(getattr(prefill, name))

    def host(cache):
        if fmt == "kv4":
            k, v = (OC.decode(x.cpu().numpy(), s.cpu().numpy()) for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
        else:
            k, v = cache.k.double().cpu().numpy(), cache.v.double().cpu().numpy()
        return k, v, cache.ctx_lens.cpu().numpy().copy(), cache.weights.double().cpu().numpy()

    for r in range(rounds):
        cache, other = caches
        k, v, lens, w = host(cache)
        par = np.stack([WT.best_first_tree(n, 15, (1, 2, 4), vocab, (r, i))[0] for i in range(b)])
        tok = np.stack([WT.best_first_tree(n, 15, (1, 2, 4), vocab, (r, i))[1] for i in range(b)])
        q, kn, vn = normal(b, n, hq, d).to(dt), normal(b, n, hkv, d).to(dt), normal(b, n, hkv, d).to(dt)
        logits = normal(b, n, vocab)
        for i in range(b):  # accept a few tokens: each node's first child
            for c in range(n - 1, 0, -1):
                logits[i, par[i, c], :] = 0
                logits[i, par[i, c], tok[i, c]] = 9.0
        dq, dkn, dvn, dpar, dtok = q.cuda(), kn.cuda(), vn.cuda(), torch.tensor(par).cuda(), torch.tensor(tok).cuda()
        out, lse = G.glance_cache_tree_verify_attn(dq, cache, dkn, dvn, dpar, sinks, window)
        acc = G.glance_greedy_accept(logits.cuda(), dpar, dtok, path_stride=16)
        G.glance_cache_weigh(dq, cache, lse, dkn, acc["accept_len"], acc["accept_path"], 0.9, sinks, window)
        G.glance_cache_commit_path(cache, dkn, dvn, acc["accept_len"], acc["accept_path"])
        kept = G.glance_cache_evict(cache, other, budget, sinks, recent)
        torch.cuda.synchronize()
        ref = OC.attention(q.double(), k, v, kn.double(), vn.double(), lens, par, sinks, window)
        assert_close(_np(out), _np(lse), *ref, dtype, f"round {r}")
        alen, path = acc["accept_len"].cpu().numpy(), acc["accept_path"].cpu().numpy()
        assert alen.min() >= 1
        wref = OC.weigh(q.double(), k, lse.double().cpu(), lens, w, 0.9, kn.double(), alen, path, sinks, window)
        now = [min(int(x) + int(a) + 1, cap) for x, a in zip(lens, alen)]
        assert cache.ctx_lens.cpu().tolist() == now
        k2, v2, lens2, w2 = host(cache)
        for i in range(b):
            np.testing.assert_allclose(w2[i, :, :now[i]], wref[i, :, :now[i]], rtol=1e-4)
        want = OC.evict(lens2, w2, budget, sinks, recent)
        ko, vo, lo, wo = host(other)
        assert lo.tolist() == [min(x, budget) for x in now]
        for i in range(b):
            for h in range(hkv):
                assert kept[i, h].cpu().tolist()[:len(want[i][h])] == want[i][h]
                np.testing.assert_array_equal(ko[i, h, :lo[i]], k2[i, h, want[i][h]])
                np.testing.assert_array_equal(vo[i, h, :lo[i]], v2[i, h, want[i][h]])
                np.testing.assert_array_equal(wo[i, h, :lo[i]], w2[i, h, want[i][h]])
        caches = [other, cache]


@pytest.mark.parametrize("fmt,dtype", [("dense", "bf16"), ("kv4", "bf16"), ("dense", "f32"), ("kv4", "f32")])
def test_rounds_of_verify_accept_weigh_commit_evict(fmt, dtype):
    _rounds(fmt, dtype)


def _pipeline(fmt):
    """Prepared calls of a round on fixed inputs, the state they change and a way to put it back."""
    c = Case("bf16", fmt, 128, 16, 8, 2, [500, 130], cap=520, seed=21, weights=True)
    q, kn, vn = c.q.cuda(), c.k_new.cuda(), c.v_new.cuda()
    lse = torch.empty(2, 16, 8, device="cuda")
    verify, out, _ = G.prepare_cache_tree_verify_attn(q, c.cache, kn, vn, c.parents.cuda(), 4, 200, lse=lse)
    draft, dout, _ = G.prepare_cache_block_draft_attn(q, c.cache, kn, vn)
    alen = torch.tensor([2, 1], dtype=torch.int32).cuda()
    path = torch.tensor([[0, 1, 2, -1], [0, 3, -1, -1]], dtype=torch.int32).cuda()
    weigh = G.prepare_cache_weigh(q, c.cache, lse, kn, alen, path, 0.5, 4, 200)
    to = G.new_cache(2, 2, 128, 128, fmt=fmt, weights=True)
    evict, kept = G.prepare_cache_evict(c.cache, to, 128, 4, 16)
    start = c.cache.weights.clone()

    def run():
        c.cache.weights.copy_(start)
        verify()
        draft()
        weigh()
        evict()

    return run, [out, dout, lse, c.cache.weights, kept, to.k, to.v, to.weights, to.ctx_lens], (c, to, q, kn, vn, alen, path)


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_captured_and_replayed(fmt):
    run, state, keep = _pipeline(fmt)
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in state]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run2, state2, keep2 = _pipeline(fmt)  # calls prepared for this stream
        run2()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run2()
    for _ in range(3):
        for t in state2:
            t.zero_()
        keep2[0].cache.weights.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, state2):
            assert torch.equal(a, b)
        run()  # eager work between the replays
        torch.cuda.synchronize()


def test_on_another_stream():
    """Calls given a stream run on it: outputs are there once it is."""
    c = Case("bf16", "kv4", 64, 8, 4, 2, [300, 200], cap=320, seed=30, weights=True)
    want = c.attn(True, 2, 100)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q, kn, vn, par = c.q.cuda(), c.k_new.cuda(), c.v_new.cuda(), c.parents.cuda()
    into = torch.zeros_like(c.cache.weights)
    torch.cuda.synchronize()  # what the current stream wrote, `into` too, is there before the other one starts
    out, lse = G.glance_cache_tree_verify_attn(q, c.cache, kn, vn, par, 2, 100, stream=s)
    w = G.glance_cache_weigh(q, c.cache, lse, n_sinks=2, window=100, weights_out=into, stream=s)
    s.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert w.sum() > 0


def test_same_bits_every_time():
    c = Case("bf16", "kv4", 128, 30, 8, 2, [900, 333], seed=31, weights=True)
    a, b = c.attn(True, 4, 500), c.attn(True, 4, 500)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    w = [G.glance_cache_weigh(c.q.cuda(), c.cache, a[1], n_sinks=4, window=500, weights_out=torch.zeros_like(c.cache.weights)) for _ in range(2)]
    assert torch.equal(w[0], w[1])


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype,d,n", [("bf16", 128, 16), ("bf16", 64, 64), ("bf16", 128, 64), ("f32", 64, 16), ("f32", 128, 40)])
def test_whole_dense_cache_is_the_plain_call(dtype, d, n, tree):
    """A dense cache without a window: the plain entry point's bits, also where the softmax's reference moves often."""
    for lens, sharp in (([1300, 77, 0], 8.0), ([2600], 1.0)):
        c = Case(dtype, "dense", d, n, 28, 4, lens, seed=51, sharp=sharp, poison=True)
        got = c.attn(tree)
        args = [t.cuda() for t in (c.q, c.cache.k, c.cache.v, c.k_new, c.v_new, c.cache.ctx_lens)]
        want = G.glance_tree_verify_attn(*args, c.parents.cuda()) if tree else G.glance_block_draft_attn(*args)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (lens, sharp)


# ------------------------------------------------------------- values and calls at the edges
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_the_smallest_values(dtype, d):
    """Around 2^-127, half the smallest code's value at the least exponent, inputs are subnormal: those above it
    round to a code that is not 0."""
    g = torch.Generator().manual_seed(d)
    rows = 96
    x = torch.exp2(torch.rand(rows, d, generator=g).double() * 10 - 131)  # 2^-131 .. 2^-121
    x[:32] = x[:32].clamp(max=2.0 ** -126)                                # blocks of subnormals alone
    step = 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149                # of the type's subnormals
    at = torch.tensor([2.0 ** -127 + i * step for i in (-1, 0, 1)] + [2.0 ** -126, 2.0 ** -126 - step, step, 3 * 2.0 ** -127, 2.0 ** -125])
    x[0, :8], x[1, :8], x[40, 8:16] = at, at[:1], at
    x = torch.where(torch.rand(rows, d, generator=g) < 0.5, x, -x).to(DT[dtype])
    assert (x != 0).sum() > x.numel() // 2 and (x.double().abs() < 2.0 ** -126).any()
    codes, scales = OC.encode(x.double())
    assert (((codes & 7) == 1) & (x.double().abs().numpy() < 2.0 ** -126)).any()
    src = G.ContextCache(x.reshape(1, 2, -1, d).cuda(), x.flip(0).reshape(1, 2, -1, d).cuda(),
                         torch.tensor([rows // 2], dtype=torch.int32).cuda())
    packed, back = G.new_cache(1, 2, rows // 2, d, fmt="kv4"), G.new_cache(1, 2, rows // 2, d, dtype=DT[dtype])
    G.glance_cache_convert(src, packed)
    G.glance_cache_convert(packed, back)
    # committed rows are rounded alike: rows 0 .. 31 of head 0 as 32 nodes of one KV head
    into = G.new_cache(1, 1, 32, d, fmt="kv4")
    new = x[:32].reshape(1, 32, 1, d).cuda()
    path = torch.arange(32, dtype=torch.int32)[None].cuda()
    G.glance_cache_commit_path(into, new, new, torch.tensor([31], dtype=torch.int32).cuda(), path)
    torch.cuda.synchronize()
    for name, ref, sc in (("k", codes, scales), ("v", codes[::-1], scales[::-1])):
        assert np.array_equal(getattr(packed, name + "_scale").cpu().numpy().reshape(rows, -1), sc)
        assert np.array_equal(getattr(packed, name).cpu().numpy().reshape(rows, -1), OC.pack(ref))
        np.testing.assert_array_equal(_np(getattr(back, name)).reshape(rows, d), OC.decode(OC.pack(ref), sc).astype(np.float32))
    assert np.array_equal(into.k.cpu().numpy().reshape(32, -1), OC.pack(codes[:32]))
    assert np.array_equal(into.v_scale.cpu().numpy().reshape(32, -1), scales[:32])


def _weigh_close(c, got, lse, ref, rows, upto, cap_fill=None):
    c.k64 = np.nan_to_num(c.k64)  # (what no row sees enters no weight)
    for b, end in enumerate(upto):
        bound = _weight_bound(c, lse.numpy(), rows, ref[b, :, :end])
        assert (np.abs(got[b, :, :end] - ref[b, :, :end]) <= bound).all(), (b, np.abs(got[b, :, :end] - ref[b, :, :end]).max())
        if cap_fill is not None:
            assert (got[b, :, end:] == cap_fill).all()


@pytest.mark.parametrize("n_sinks,window", [(0, 1), (3, 1), (5, 40), (70, 100), (1, 190)])
@pytest.mark.parametrize("fmt,dtype,d", [("dense", "bf16", 128), ("kv4", "bf16", 64), ("dense", "f32", 64), ("kv4", "f32", 128)])
def test_weights_do_not_depend_on_unseen_slots(fmt, dtype, d, n_sinks, window):
    """NaN in every slot that no row sees: those slots only fade."""
    lens = [0, 1, 40, 64, 65, 200, 321]
    c = Case(dtype, fmt, d, 9, 4, 2, lens, cap=330, seed=window + d, poison=True, n_sinks=n_sinks, window=window, weights=True)
    lse = torch.tensor(c.want(False, n_sinks, window)[1], dtype=torch.float32)
    into = torch.full_like(c.cache.weights, 7.0)
    got = G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=0.5, n_sinks=n_sinks, window=window, weights_out=into).cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref = OC.weigh(c.q.double(), c.k64, lse.double(), c.lens, c.weights.double(), 0.5, n_sinks=n_sinks, window=window)
    assert np.isfinite(ref).all()
    _weigh_close(c, got, lse, ref, 18, lens, 7.0)


@pytest.mark.parametrize("n_sinks,window", [(0, 0), (5, 40)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt,dtype", [("dense", "bf16"), ("kv4", "bf16"), ("dense", "f32"), ("kv4", "f32")])
def test_weights_of_the_longest_path(fmt, dtype, d, n_sinks, window):
    """A path of 64 nodes of 14 heads: more rows than a workgroup holds at a time, and slots-to-be past the capacity."""
    lens, cap = [300, 0, 680], 700
    c = Case(dtype, fmt, d, 64, 14, 1, lens, cap=cap, seed=d, weights=True)
    c.parents = torch.arange(-1, 63, dtype=torch.int32).repeat(3, 1)
    lse = torch.tensor(c.want(True, n_sinks, window)[1], dtype=torch.float32)
    alen, path = torch.tensor([63, 63, 2 ** 31 - 1], dtype=torch.int32), torch.arange(64, dtype=torch.int32).repeat(3, 1)
    into = torch.full_like(c.cache.weights, 7.0)
    got = G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), c.k_new.cuda(), alen.cuda(), path.cuda(), 0.5, n_sinks, window, into).cpu().numpy()
    ref = OC.weigh(c.q.double(), c.k64, lse.double(), c.lens, c.weights.double(), 0.5, c.k_new.double().numpy(), alen.numpy(), path.numpy(),
                   n_sinks, window)
    _weigh_close(c, got, lse, ref, 64 * 14, [364, 64, cap], 7.0)


@pytest.mark.parametrize("fmt,dtype", [("dense", "bf16"), ("kv4", "f32")])
def test_weights_from_none(fmt, dtype):
    """With decay 0 the cache needs no weights; without any an output has to be given."""
    c = Case(dtype, fmt, 64, 5, 4, 2, [90, 3], seed=8)
    lse = torch.tensor(c.want(False)[1], dtype=torch.float32)
    with pytest.raises(ValueError, match="weights"):
        G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=0.0)
    into = torch.full((2, 2, 90), float("nan")).cuda()
    with pytest.raises(G.GlanceError, match="weights"):
        G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=0.5, weights_out=into)
    got = G.glance_cache_weigh(c.q.cuda(), c.cache, lse.cuda(), decay=0.0, weights_out=into).cpu().numpy()
    ref = OC.weigh(c.q.double(), c.k64, lse.double(), c.lens, np.zeros((2, 2, 90)), 0.0)
    _weigh_close(c, got, lse, ref, 10, [90, 3])
    assert np.isnan(got[1, :, 3:]).all()


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_every_call_clamps_lengths(fmt):
    """Lengths below 0 and past the capacity give what 0 and the capacity give."""
    outs = []
    for lens in ([120, 0, 64], [10 ** 9, -5, 64]):
        c = Case("bf16", fmt, 64, 4, 4, 2, [120, 0, 64], cap=120, seed=17, weights=True)
        c.cache.ctx_lens = torch.tensor(lens, dtype=torch.int32).cuda()
        q, kn, vn = c.q.cuda(), c.k_new.cuda(), c.v_new.cuda()
        lse = torch.ones(3, 4, 4).cuda()
        got = [G.glance_cache_weigh(q, c.cache, lse, decay=0.5, n_sinks=3, window=50, weights_out=torch.zeros(3, 2, 120).cuda())]
        to = G.new_cache(3, 2, 70, 64, fmt=fmt, weights=True)
        got += [G.glance_cache_evict(c.cache, to, 70, 3, 5), to.k, to.v, to.weights, to.ctx_lens]
        other = G.new_cache(3, 2, 100, 64, fmt="dense" if fmt == "kv4" else "kv4")
        G.glance_cache_convert(c.cache, other)
        got += [other.k, other.v, other.ctx_lens]
        path = torch.tensor([[0, 2, -1]] * 3, dtype=torch.int32).cuda()
        G.glance_cache_commit_path(c.cache, kn, vn, torch.tensor([1, 1, 1], dtype=torch.int32).cuda(), path)
        got += [c.cache.k, c.cache.v, c.cache.ctx_lens]
        torch.cuda.synchronize()
        outs.append(got)
    assert outs[1][5].cpu().tolist() == [70, 0, 64] and outs[1][-1].cpu().tolist() == [120, 2, 66]
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_calls_on_another_stream_give_the_same(fmt):
    """Every call that takes a stream, on one of its own: the bits of the same calls on the current stream."""
    def results(stream):
        c = Case("bf16", fmt, 64, 8, 4, 2, [300, 200], cap=320, seed=30, weights=True)
        q, kn, vn, par = c.q.cuda(), c.k_new.cuda(), c.v_new.cuda(), c.parents.cuda()
        alen = torch.tensor([2, 1], dtype=torch.int32).cuda()
        path = torch.tensor([[0, 1, 2], [0, 1, -1]], dtype=torch.int32).cuda()
        into = torch.zeros_like(c.cache.weights)
        to = G.new_cache(2, 2, 128, 64, fmt=fmt, weights=True)
        other = G.new_cache(2, 2, 320, 64, fmt="dense" if fmt == "kv4" else "kv4")
        torch.cuda.synchronize()  # all of it is there before a stream of the calls' own starts
        out, lse = G.glance_cache_tree_verify_attn(q, c.cache, kn, vn, par, 2, 100, stream=stream)
        draft = G.glance_cache_block_draft_attn(q, c.cache, kn, vn, stream=stream)
        G.glance_cache_weigh(q, c.cache, lse, kn, alen, path, 0.5, 2, 100, weights_out=into, stream=stream)
        G.glance_cache_commit_path(c.cache, kn, vn, alen, path, stream=stream)
        kept = G.glance_cache_evict(c.cache, to, 128, 2, 16, stream=stream)
        G.glance_cache_convert(c.cache, other, stream=stream)
        torch.cuda.synchronize()
        return [out, lse, *draft, into, c.cache.k, c.cache.ctx_lens, kept, to.k, to.v, to.weights, to.ctx_lens, other.k, other.v,
                other.ctx_lens]

    want = results(None)
    assert (want[4] > 0).any()
    for a, b in zip(results(torch.cuda.Stream()), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_rounds_on_a_stream_of_their_own(fmt):
    with torch.cuda.stream(torch.cuda.Stream()):
        _rounds(fmt, "bf16", rounds=2)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_conversion_and_commit_captured(dtype):
    """A prepared conversion both ways and a commit between them, replayed with other work between the replays."""
    c = Case(dtype, "dense", 64, 6, 2, 2, [40, 9], cap=48, seed=41)
    kn, vn = c.k_new.cuda(), c.v_new.cuda()
    alen, path = torch.tensor([2, 0], dtype=torch.int32).cuda(), torch.tensor([[0, 3, 5], [1, -1, -1]], dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    packed, back = G.new_cache(2, 2, 48, 64, fmt="kv4"), G.new_cache(2, 2, 48, 64, dtype=DT[dtype])
    pack, unpack = (G.prepare_cache_convert(a, b, stream=side) for a, b in ((c.cache, packed), (packed, back)))
    state = [packed.k, packed.v, packed.k_scale, packed.v_scale, packed.ctx_lens, back.k, back.v, back.ctx_lens]

    def run():
        pack()
        G.glance_cache_commit_path(packed, kn, vn, alen, path, stream=side)
        unpack()

    torch.cuda.synchronize()
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in state]
    assert want[4].cpu().tolist() == [43, 10]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for _ in range(3):
        for t in state:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(state, want):
            assert torch.equal(a, b)
        run()
        torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["dense", "kv4"])
def test_evict_past_32_bits_from_every_head(fmt):
    """Kept slots over a whole cache of more than 4 GB a side: each head's known ones, in order, with their rows."""
    hkv, cap, d, some, sinks, recent = (2, 2 ** 24 + 3, 128, 300, 8, 12) if fmt == "dense" else (4, 2 ** 25, 128, 300, 8, 12)
    rng = np.random.default_rng(1)
    slots = [np.sort(rng.permutation(np.unique(rng.integers(sinks, cap - recent, 2 * some)))[:some]) for _ in range(hkv)]
    src = G.new_cache(1, hkv, cap, d, fmt=fmt, weights=True)
    src.ctx_lens.fill_(cap)
    want = []
    for g in range(hkv):
        at = torch.tensor(slots[g]).cuda()
        src.weights[0, g, at] = torch.arange(1, some + 1, dtype=torch.float32).cuda()
        keep = np.concatenate([np.arange(sinks), slots[g], np.arange(cap - recent, cap)])
        want.append(keep.tolist())
        at = torch.tensor(keep).cuda()
        for i, t in enumerate((src.k, src.v)):  # rows that tell their slot and side
            t[0, g, at, :4] = torch.stack([(at >> s) % 16 + i for s in (0, 4, 8, 12)], -1).to(t.dtype)
    to = G.new_cache(1, hkv, some + sinks + recent, d, fmt=fmt, weights=True)
    kept = G.glance_cache_evict(src, to, some + sinks + recent, sinks, recent)
    torch.cuda.synchronize()
    assert to.ctx_lens.item() == some + sinks + recent
    for g in range(hkv):
        assert kept[0, g].cpu().tolist() == want[g]
        at = torch.tensor(want[g]).cuda()
        for t, s in ((to.k, src.k), (to.v, src.v), (to.weights, src.weights)):
            assert torch.equal(t[0, g], s[0, g, at])


@pytest.mark.parametrize("fmt,n_sinks,window", [("dense", 4, 1500), ("dense", 0, 0), ("kv4", 0, 0), ("kv4", 9, 700)])
@pytest.mark.parametrize("n", [1, 16, 64])
def test_bf16_outputs_err_by_two_roundings(fmt, n_sinks, window, n):
    """Probabilities are rounded to bf16 before P.V and outputs once more.  Derived: with values independent of mean 0
    an output is sqrt(sum w^2) of theirs in size and the error of the first rounding at most 2^-8 / sqrt(3) of that
    (each probability's error is spread over half a step either way, at most 2^-8 of it), of the second the same, of a
    piece's fp16 2^-11 / sqrt(3): the root of their squares is 3.2e-3.  Nothing else enters."""
    c = Case("bf16", fmt, 128, n, 28, 4, [2048, 1777], seed=60 + n)
    out, _ = c.attn(True, n_sinks, window)
    ref = c.want(True, n_sinks, window)[0]
    assert np.sqrt(((_np(out) - ref) ** 2).mean() / (ref ** 2).mean()) < 3.3e-3
