"""The paged KV cache on the GPU: appending, reading back, decoding, against plain forms in 64 bits.

Everything that a call must not look at -- rows of a last page behind the sequence, pages of nobody, scales of such pages -- holds
NaN, and everything that it must not write is compared afterwards.
"""
import math

import numpy as np
import pytest
import torch

from paper_2608_19758_b200 import binding

pytestmark = pytest.mark.gpu
D = 128
E4M3 = torch.float8_e4m3fn
SCALE = 1.0 / math.sqrt(D)


def e4m3_values():
    v = torch.arange(256, dtype=torch.uint8).view(E4M3).double()
    return v


def nearest_e4m3(x):
    """Bytes of the e4m3 values nearest to x (64 bits), ties to the even code, saturating; NaN stays NaN."""
    pos = e4m3_values()[:127].numpy()                      # 0 .. 448 ascending, code = index
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    mid = (pos[lo] + pos[hi]) / 2
    code = np.where((a > mid) | ((a == mid) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(x), 127, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


class Store:
    """A cache with its pages handed out at random; K, V and scales as 64-bit values by token for the plain form."""

    def __init__(self, fmt, lens, hq, hkv, page, seed=0, spare=3, capacity=None, fill=True, spread=2):
        self.fmt, self.lens, self.hq, self.hkv, self.page = fmt, list(lens), hq, hkv, page
        rng = self.rng = np.random.default_rng(seed)
        cap = [max(a, b) for a, b in zip(lens, capacity or lens)]
        need = [-(-n // page) for n in cap]
        self.pool, self.mp = sum(need) + spare, max(max(need), 1)
        ids = rng.permutation(self.pool)
        self.pt = np.full((len(lens), self.mp), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.pt[b, :n] = ids[at:at + n]
            at += n
        self.cache = binding.Cache(dict(max_seqs=max(len(lens), 1), num_q_heads=hq, num_kv_heads=hkv, head_dim=D, page_size=page,
                                        num_pages=self.pool, max_pages_per_seq=self.mp, format=fmt, softmax_scale=0.0))
        shape = (self.pool, page, hkv, D)
        self.ks = self.vs = None
        if fmt == 0:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=torch.bfloat16) for _ in "kv")
        else:
            self.k, self.v = (torch.full(shape, 0x7F, dtype=torch.uint8) for _ in "kv")
            if fmt == 1:
                self.ks, self.vs = (torch.from_numpy(np.exp(rng.normal(-4, 0.3, hkv))).float() for _ in "kv")
            else:
                self.ks, self.vs = (torch.full((self.pool, hkv), float("nan")) for _ in "kv")
        if fill:
            for b, n in enumerate(lens):
                for t in range(-(-n // page)):
                    pid, rows = self.pt[b, t], min(page, n - t * page)
                    for x, s in ((self.k, self.ks), (self.v, self.vs)):
                        val = torch.from_numpy(rng.normal(0, 1, (rows, hkv, D)))
                        if fmt == 0:
                            x[pid, :rows] = val.bfloat16()
                        else:
                            x[pid, :rows] = (val * 60).to(torch.float32).clamp(-448, 448).to(E4M3).view(torch.uint8)
                            if fmt == 2:      # pages of unlike size, not all of them powers of two
                                s[pid] = torch.from_numpy(np.exp2(rng.integers(-6 - spread, -5 + spread, hkv)) * (1 + (pid % 3) / 4)).float()
        self.to_gpu()

    def to_gpu(self):
        g = lambda t: None if t is None else t.cuda()
        self.dk, self.dv, self.dks, self.dvs = g(self.k), g(self.v), g(self.ks), g(self.vs)
        self.dpt = torch.from_numpy(self.pt).cuda()
        self.ws = self.cache.new_workspace()

    def tokens(self, b, n=None):
        """K, V of sequence b in 64 bits [n, hkv, D], from the GPU's copy."""
        n = self.lens[b] if n is None else n
        out = []
        for x, s in ((self.dk, self.dks), (self.dv, self.dvs)):
            pid = torch.from_numpy(self.pt[b, np.arange(n) // self.page].astype(np.int64))
            row = torch.arange(n) % self.page
            x = x.cpu()[pid, row]
            x = x.double() if self.fmt == 0 else x.view(E4M3).double()
            if self.fmt == 1:
                x = x * s.cpu().double()[:, None]
            elif self.fmt == 2:
                x = x * s.cpu().double()[pid][:, :, None]
            out.append(x)
        return out

    def decode(self, q, lq, window=0, sinks=0, lens=None, out=None, lse=None, stream=None, ws=None):
        cu = torch.tensor(np.concatenate([[0], np.cumsum(lq)]), dtype=torch.int32).cuda()
        lk = torch.tensor(self.lens if lens is None else lens, dtype=torch.int32).cuda()
        out = torch.full((q.shape[0], self.hq, D), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
        lse = torch.full((self.hq, q.shape[0]), float("nan"), device="cuda") if lse is None else lse
        binding.fp2_decode(self.cache, q, self.dk, self.dv, self.dpt, cu, lk, self.dks, self.dvs, out, lse,
                           self.ws if ws is None else ws, window_tokens=window, sink_tokens=sinks, stream=stream)
        return out, lse


def attend(q, k, v, first, window, sinks):
    """One sequence in 64 bits: out [n, hq, D], lse [hq, n], and what the tolerances need: the weighted sum of |V|, and a bound on
    sum |q k| scale."""
    n, hq, hkv, L = q.shape[0], q.shape[1], k.shape[1], k.shape[0]
    pos, key = first + torch.arange(n)[:, None], torch.arange(L)[None]
    see = key <= pos
    if window:
        see &= (pos - key < window) | (key < sinks)
    used = see.any(0)
    k, v = torch.where(used[:, None, None], k, torch.zeros_like(k)), torch.where(used[:, None, None], v, torch.zeros_like(v))
    g = hq // hkv
    out, lse, mass, size = torch.zeros(n, hq, D, dtype=torch.float64), torch.zeros(hq, n, dtype=torch.float64), torch.zeros(n, hq, D, dtype=torch.float64), 0.0
    for h in range(hq):
        x = (q[:, h].double() @ k[:, h // g].T) * SCALE
        size = max(size, float((q[:, h].double().abs() @ k[:, h // g].abs().T).max()) * SCALE) if L else size
        x = x.masked_fill(~see, -math.inf)
        lse[h] = torch.logsumexp(x, 1) if L else -math.inf
        w = torch.nan_to_num(torch.exp(x - torch.where(torch.isinf(lse[h]), torch.zeros_like(lse[h]), lse[h])[:, None]))
        out[:, h], mass[:, h] = w @ v[:, h // g], w @ v[:, h // g].abs()
    return out, lse, mass, size


def close(out, lse, q, k, v, first, window, sinks):
    """One sequence's rows against the plain form.  Logits: 128 products summed in fp32, at most 128 * 2^-24 of sum |q k| scale off,
    and a scaling and two approximate functions of 2^-22 relative each: d = (2^-17 + 2^-20) size + 2^-20.  A weight is off by that
    factor and by its rounding (BF16 pair 2^-17, F16 2^-11, and 2^-25 / 2^8 of the largest weight where F16 runs out); the sums of n
    positive terms by n 2^-24 at most.  The output is rounded once: 2^-8."""
    n = k.shape[0]
    ro, rl, mass, size = attend(q.cpu(), k, v, first, window, sinks)
    d = (2.0 ** -17 + 2.0 ** -20) * size + 2.0 ** -20 + n * 2.0 ** -24
    vmax = float(torch.nan_to_num(v).abs().max()) if n else 0.0
    tol = 2.0 ** -8 * ro.abs() + (2 * d + 2.0 ** -11 + 2.0 ** -16) * mass * (1 + 2.0 ** -8) + 2.0 ** -33 * n * vmax
    err = (out.double().cpu() - ro).abs()
    assert bool((err <= tol).all()), (n, float((err - tol).max()), float(err.max()))
    dead, lse = torch.isinf(rl), lse.double().cpu()
    assert bool((lse[dead] == -math.inf).all())
    assert bool(((lse - rl)[~dead].abs() <= d + 2.0 ** -22 * rl[~dead].abs()).all())


def check(store, q, lq, out, lse, window, sinks, lens=None):
    lens, at = store.lens if lens is None else lens, 0
    for b, n in enumerate(lq):
        if n:
            k, v = store.tokens(b, lens[b])
            close(out[at:at + n], lse[:, at:at + n], q[at:at + n], k, v, lens[b] - n, window, sinks)
        at += n


def queries(rng, n, hq, sharp=1.0):
    return torch.from_numpy(rng.normal(0, sharp, (n, hq, D))).bfloat16().cuda()


LENS = [
    ([1], [1]), ([777], [1]), ([64, 65, 63, 1, 16, 17, 128], [1] * 7), ([300, 5, 0, 1000, 40], [1, 5, 0, 3, 2]),
    ([130, 2000, 33], [0, 17, 33]), ([4096], [1]), ([515] * 40, [1] * 40),
]


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("heads,page", [((8, 2), 16), ((4, 1), 128), ((28, 4), 64), ((8, 8), 8), ((16, 1), 32), ((6, 2), 8)])
@pytest.mark.parametrize("which", range(len(LENS)))
def test_decode(fmt, heads, page, which):
    lens, lq = LENS[which]
    st = Store(fmt, lens, *heads, page, seed=which + 10 * fmt)
    q = queries(st.rng, sum(lq), heads[0], 1.5)
    for window, sinks in [(0, 0), (100, 4), (1, 0), (64, 70)]:
        out, lse = st.decode(q, lq, window, sinks)
        check(st, q, lq, out, lse, window, sinks)
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_decode_long_and_many(fmt):
    """Units cut over many CTAs and units that end inside a share, in one call; more sequences than a scan step holds."""
    rng = np.random.default_rng(5)
    lens = [20000] + [int(x) for x in rng.integers(1, 400, 200)]
    lq = [2] + [min(n, int(x)) for n, x in zip(lens[1:], rng.integers(0, 4, 200))]
    st = Store(fmt, lens, 4, 2, 16, seed=5)
    q = queries(st.rng, sum(lq), 4)
    for window, sinks in [(0, 0), (5000, 100)]:
        out, lse = st.decode(q, lq, window, sinks)
        check(st, q, lq, out, lse, window, sinks)
        for _ in range(3):   # the same bits every time, whoever arrives last
            o2, l2 = st.decode(q, lq, window, sinks)
            assert torch.equal(out.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, l2)


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_decode_extreme_sizes(fmt):
    """Sharp logits, queries of very unlike size in one tile, page scales 2^20 apart."""
    st = Store(fmt, [500, 260], 8, 2, 16, seed=9, spread=10)
    q = queries(st.rng, 3, 8)
    q = (q.float() * torch.exp2(torch.tensor([-60.0, 0, 3, -3, 5, -20, 1, 4], device="cuda"))[None, :, None]).bfloat16()
    out, lse = st.decode(q, [2, 1])
    check(st, q, [2, 1], out, lse, 0, 0)


def test_decode_hidden_places_do_not_matter():
    """Tokens in front of the windows hold NaN and infinities, their pages may be gone; rows behind the last sequence stay."""
    for fmt in (0, 1, 2):
        st = Store(fmt, [900, 333], 8, 2, 16, seed=3)
        q = queries(st.rng, 6, 8)
        lq = [2, 1]
        out, lse = (torch.full((6, 8, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((8, 6), 7.0, device="cuda"))
        clean, clean_l = st.decode(q, lq, 50, 5, out=out.clone(), lse=lse.clone())
        check(st, q, lq, clean, clean_l, 50, 5)
        assert bool((clean[3:] == 7.0).all()) and bool((clean_l[:, 3:] == 7.0).all())
        bad = float("nan")
        for b, n in enumerate(lq):
            for tok in range(5, st.lens[b] - n - 50 + 1):
                pid, row = int(st.pt[b, tok // 16]), tok % 16
                for x in (st.dk, st.dv):
                    x[pid, row] = (bad if tok % 2 else math.inf) if fmt == 0 else 0x7F
            for t in range(1, (st.lens[b] - n - 50 + 1) // 16):     # pages wholly in front of the windows, behind the sinks
                st.dpt[b, t] = -1 if t % 2 else st.pool + 5
                if fmt == 2:
                    st.dks[int(st.pt[b, t])] = bad
        got, got_l = st.decode(q, lq, 50, 5, out=out.clone(), lse=lse.clone())
        assert torch.equal(got.view(torch.int16), clean.view(torch.int16)) and torch.equal(got_l, clean_l)
        assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


def test_decode_reports_and_skips_what_does_not_fit():
    st = Store(2, [100, 200, 64], 8, 2, 16, seed=4)
    q = queries(st.rng, 3, 8)
    good, good_l = st.decode(q, [1, 1, 1])
    # a page of sequence 1 outside the pool: its tokens are left out, the others as before
    st.dpt[1, 3] = st.pool
    out, lse = st.decode(q, [1, 1, 1])
    code, words = binding.fp2_cache_read_status(st.cache, st.ws, raise_on_error=False)
    assert code == 1 and words[2] == 2
    assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    k, v = st.tokens(1)
    keep = [t for t in range(200) if t // 16 != 3]
    close(out[1:2], lse[:, 1:2], q[1:2], k[keep], v[keep], len(keep) - 1, 0, 0)
    st.dpt[1, 3] = int(st.pt[1, 3])
    # lengths that do not fit: the sequence's rows are not written
    for cu, lens in [([0, 1, 2, 3], [100, 10 ** 6, 64]), ([0, 1, -1, 3], [100, 200, 64]), ([0, 1, 9, 3], [100, 200, 64]), ([0, 1, 2, 3], [100, -5, 64])]:
        out = torch.full_like(good, 3.0)
        binding.fp2_decode(st.cache, q, st.dk, st.dv, st.dpt, torch.tensor(cu, dtype=torch.int32).cuda(),
                           torch.tensor(lens, dtype=torch.int32).cuda(), st.dks, st.dvs, out, None, st.ws)
        code, words = binding.fp2_cache_read_status(st.cache, st.ws, raise_on_error=False)
        assert code == 1 and words[2] == 4
        assert torch.equal(out[0], good[0]) and bool((out[1] == 3.0).all())
    # more queries than tokens: the first ones stand in front of the sequence and see nothing
    st2 = Store(2, [2], 8, 2, 16, seed=4)
    q2 = queries(st2.rng, 5, 8)
    out, lse = st2.decode(q2, [5])
    check(st2, q2, [5], out, lse, 0, 0)
    assert bool((out[:3] == 0).all()) and bool((lse[:, :3] == -math.inf).all())
    out, lse = st2.decode(q2[:1], [1], lens=[0])
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_decode_query_strides_streams_and_graphs():
    """Queries as slices of a fused projection; a side stream with a workspace of its own; a captured call replayed while the
    sequences grow."""
    st = Store(2, [300, 40, 1000], 8, 2, 32, seed=6, capacity=[400, 64, 1100])
    fused = torch.randn(3, 8 * D + 512, device="cuda").bfloat16()
    q = fused[:, :8 * D].view(3, 8, D)
    out, lse = st.decode(q, [1, 1, 1])
    check(st, q.contiguous(), [1, 1, 1], out, lse, 0, 0)
    side, ws2 = torch.cuda.Stream(), st.cache.new_workspace()
    torch.cuda.synchronize()
    outs = []
    for k in range(6):
        outs.append(st.decode(q, [1, 1, 1], stream=side if k % 2 else None, ws=ws2 if k % 2 else st.ws))
    torch.cuda.synchronize()
    assert all(torch.equal(o, out) and torch.equal(l, lse) for o, l in outs)
    # capture append + decode, replay with longer sequences
    cu = torch.tensor([0, 1, 2, 3], dtype=torch.int32).cuda()
    lk = torch.tensor([300, 40, 1000], dtype=torch.int32).cuda()
    new = torch.zeros(3, 2, 2, D, dtype=torch.bfloat16, device="cuda")
    qs, out = torch.zeros(3, 8, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 8, D, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(8, 3, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lk += 1
        binding.fp2_cache_append(st.cache, new[:, 0], new[:, 1], st.dpt, cu, lk, st.dk, st.dv, st.dks, st.dvs, st.ws)
        binding.fp2_decode(st.cache, qs, st.dk, st.dv, st.dpt, cu, lk, st.dks, st.dvs, out, lse, st.ws)
    for step in range(1, 24):
        new.copy_(torch.randn_like(new))
        qs.copy_(torch.randn_like(qs))
        graph.replay()
        if step in (1, 2, 7, 23):
            check(st, qs, [1, 1, 1], out, lse, 0, 0, lens=[300 + step, 40 + step, 1000 + step])
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


def test_decode_without_lse_and_with_nothing_to_do():
    st = Store(1, [50, 60], 8, 2, 16)
    q = queries(st.rng, 2, 8)
    out, _ = st.decode(q, [1, 1])
    o2 = torch.empty_like(out)
    cu, lk = torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), torch.tensor([50, 60], dtype=torch.int32).cuda()
    binding.fp2_decode(st.cache, q, st.dk, st.dv, st.dpt, cu, lk, st.dks, st.dvs, o2, None, st.ws)
    assert torch.equal(out, o2)
    binding.fp2_decode(st.cache, q[:0], st.dk, st.dv, st.dpt, cu, lk, st.dks, st.dvs, o2[:0], None, st.ws)
    cu.zero_()     # sequences without queries: nothing is written
    o2.fill_(5.0)
    binding.fp2_decode(st.cache, q, st.dk, st.dv, st.dpt, cu, lk, st.dks, st.dvs, o2, None, st.ws)
    assert bool((o2 == 5.0).all())


# ---------------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------------
def page_scale(amax):
    return max(2.0 ** math.ceil(math.log2(amax / 448)), 2.0 ** -100) if amax > 0 else 2.0 ** -100


def plain_append(st, x, lens, news, name):
    """The cache and scales after the append, from the definition: bytes (or BF16 values) and fp32 scales."""
    cache = (st.dk if name == "k" else st.dv).cpu().clone()
    scale = (st.dks if name == "k" else st.dvs)
    scale = None if scale is None else scale.cpu().clone()
    x, at = x.cpu(), 0
    for b, n in enumerate(news):
        first = lens[b] - n
        for t in range(first // st.page, -(-lens[b] // st.page)) if n else ():
            pid, lo, hi = int(st.pt[b, t]), max(first, t * st.page), min(lens[b], (t + 1) * st.page)
            rows = x[at + lo - first:at + hi - first]
            lo, hi = lo - t * st.page, hi - t * st.page
            if st.fmt == 0:
                cache[pid, lo:hi] = rows
                continue
            for h in range(st.hkv):
                r = rows[:, h].double().numpy()
                if st.fmt == 1:
                    s = np.float32(scale[h])
                    r = (rows[:, h].float().numpy() / s).astype(np.float64)     # the quotient as the call takes it, in 32 bits
                else:
                    fin = np.abs(r[np.isfinite(r)])
                    s = page_scale(fin.max() if fin.size else 0.0)
                    if lo:
                        before = float(scale[pid, h])
                        s = max(s, before)
                        if s > before:
                            old = cache[pid, :lo, h].view(E4M3).double().numpy()
                            cache[pid, :lo, h] = torch.from_numpy(nearest_e4m3((old.astype(np.float32) * np.float32(before)).astype(np.float64) / s))
                    scale[pid, h] = s
                    r = (r.astype(np.float32) / np.float32(s)).astype(np.float64)
                cache[pid, lo:hi, h] = torch.from_numpy(nearest_e4m3(np.clip(r, -448, 448)))
        at += n
    return cache, scale


def run_append(st, k_new, v_new, lens, news):
    cu = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32).cuda()
    lk = torch.tensor(lens, dtype=torch.int32).cuda()
    binding.fp2_cache_append(st.cache, k_new, v_new, st.dpt, cu, lk, st.dk, st.dv, st.dks, st.dvs, st.ws)


def same(a, b):
    """Bit for bit, NaN scales of pages of nobody included."""
    if a is None:
        return b is None
    a, b = a.cpu().contiguous(), b.cpu().contiguous()
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.view(kind), b.view(kind))


APPENDS = [
    ([0], [1]), ([776], [1]), ([0, 0, 0], [1, 130, 16]), ([5, 16, 17, 0, 300], [1, 1, 40, 0, 129]), ([127, 128, 1, 0], [1, 2, 126, 500]),
    (list(range(70)), [1] * 70),
]


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("hkv,page", [(2, 16), (1, 128), (4, 64), (8, 8), (3, 32)])
@pytest.mark.parametrize("which", range(len(APPENDS)))
def test_append(fmt, hkv, page, which):
    had, news = APPENDS[which]
    lens = [a + n for a, n in zip(had, news)]
    st = Store(fmt, had, hkv, hkv, page, seed=which, capacity=lens)
    total = sum(news)
    fused = torch.from_numpy(st.rng.normal(0, 1, (total + 2, 3 * hkv * D))).bfloat16().cuda()    # (two rows behind the last)
    fused *= torch.exp2(torch.from_numpy(st.rng.integers(-9, 9, (total + 2, 1)))).bfloat16().cuda()
    fused[total // 2, :2 * D] = 0.0
    k_new, v_new = fused[:, :hkv * D].view(-1, hkv, D), fused[:, 2 * hkv * D:].view(-1, hkv, D)
    want = plain_append(st, k_new, lens, news, "k") + plain_append(st, v_new, lens, news, "v")
    run_append(st, k_new, v_new, lens, news)
    for got, ref in zip((st.dk, st.dks, st.dv, st.dvs), want):
        assert same(got, ref)
    run_append(st, k_new, v_new, lens, news)      # again: the same (the scales are there already)
    for got, ref in zip((st.dk, st.dks, st.dv, st.dvs), want):
        assert same(got, ref)
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


def test_append_values_that_are_not_finite():
    for fmt in (1, 2):
        st = Store(fmt, [0], 2, 2, 16, capacity=[20])
        x = torch.from_numpy(st.rng.normal(0, 1, (20, 2, D))).bfloat16()
        x[3, 0, 5], x[4, 0, 6], x[4, 1, 7] = math.nan, math.inf, -math.inf
        x[16:, 1] = 0.0                       # a page whose head has nothing but zeros and infinities
        x[17, 1, 3] = -math.inf
        x = x.cuda()
        want = plain_append(st, x, [20], [20], "k")
        run_append(st, x, x, [20], [20])
        assert same(st.dk, want[0]) and same(st.dks, want[1])
        got = st.dk.cpu()[int(st.pt[0, 0])]
        assert got[3, 0, 5] & 0x7F == 0x7F and got[4, 0, 6] == 0x7E and got[4, 1, 7] == 0xFE
        if fmt == 2:
            assert float(st.dks[int(st.pt[0, 1]), 1]) == 2.0 ** -100


def test_append_smallest_and_largest_numbers():
    """Scales at the ends of their range: BF16 subnormals go to the floor 2^-100, the largest finite value needs 2^120."""
    st = Store(2, [0], 1, 1, 16, capacity=[48])
    x = torch.zeros(48, 1, D, dtype=torch.bfloat16)
    x[:16] = 2.0 ** -130
    x[16:32] = torch.finfo(torch.bfloat16).max
    x[32:, 0, :] = torch.tensor([448.0, 449.0, 1.75 * 2 ** -30, 1.76 * 2 ** -30] * 32).bfloat16()[None]
    x = x.cuda()
    want = plain_append(st, x, [48], [48], "k")
    run_append(st, x, x, [48], [48])
    assert same(st.dk, want[0]) and same(st.dks, want[1]) and same(st.dv, want[0])
    s = [float(st.dks[int(st.pt[0, t]), 0]) for t in range(3)]
    assert s[0] == 2.0 ** -100 and s[1] == 2.0 ** 120 and s[2] == 1.0


def test_append_token_by_token_ends_where_one_call_does():
    """Growing scales: the page ends with the scale it would have got at once, and with the same values wherever the e4m3 value is
    normal under it; below that a value was rounded at every growth, each time by half a step of 2^-9 of the scale then."""
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.normal(0, 1, (40, 2, D)) * np.exp2(rng.uniform(-4, 4, (40, 1, 1)))).bfloat16().cuda()
    one, each = (Store(2, [0], 2, 2, 16, capacity=[40]) for _ in "ab")
    run_append(one, x, x, [40], [40])
    for t in range(40):
        run_append(each, x[t:t + 1], x[t:t + 1], [t + 1], [1])
    ids = one.pt[0, :3].astype(np.int64)
    assert np.array_equal(each.pt[0, :3], one.pt[0, :3])
    assert torch.equal(one.dks[ids], each.dks[ids]) and torch.equal(one.dvs[ids], each.dvs[ids])
    a, b = one.dk[ids].view(E4M3).float()[:2].cpu(), each.dk[ids].view(E4M3).float()[:2].cpu()
    normal = a.abs() >= 2.0 ** -6
    assert torch.equal(a[normal], b[normal]) and bool(((a - b).abs() <= 2.0 ** -9).all())


def test_append_reports_and_skips_what_does_not_fit():
    st = Store(2, [16, 16, 16], 2, 2, 16, capacity=[40, 40, 40])
    x = torch.from_numpy(st.rng.normal(0, 1, (6, 2, D))).bfloat16().cuda()
    before = st.dk.clone()
    st.dpt[1, 1] = -1
    run_append(st, x, x, [18, 18, 18], [2, 2, 2])
    code, words = binding.fp2_cache_read_status(st.cache, st.ws, raise_on_error=False)
    assert code == 1 and words[2] == 2
    changed = (st.dk != before).flatten(1).any(1).cpu().nonzero().flatten().tolist()
    assert sorted(changed) == sorted([int(st.pt[0, 1]), int(st.pt[2, 1])])
    st.dpt[1, 1] = int(st.pt[1, 1])
    for lens, cu in [([18, 1, 18], [0, 2, 4, 6]), ([18, 49, 18], [0, 2, 4, 6]), ([18, 18, 18], [0, 2, 9, 6]), ([18, 18, 18], [0, 2, 1, 6])]:
        before = st.dk.clone()
        binding.fp2_cache_append(st.cache, x * 2, x * 2, st.dpt, torch.tensor(cu, dtype=torch.int32).cuda(),
                                 torch.tensor(lens, dtype=torch.int32).cuda(), st.dk, st.dv, st.dks, st.dvs, st.ws)
        code, words = binding.fp2_cache_read_status(st.cache, st.ws, raise_on_error=False)
        assert code == 1 and words[2] == 4
        assert same(st.dk[[int(p) for p in st.pt[1]]], before[[int(p) for p in st.pt[1]]])


# ---------------------------------------------------------------------------------------------------------------------
# expand, and the calls together
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("hkv,page", [(2, 16), (1, 128), (4, 64), (8, 8), (3, 32)])
@pytest.mark.parametrize("lens", [[1], [777], [0, 16, 17, 300, 15], [64] * 35 + [0] * 5 + [129] * 30])
def test_expand(fmt, hkv, page, lens):
    st = Store(fmt, lens, hkv, hkv, page, seed=2)
    need = [-(-n // page) for n in lens]
    out_pt = np.full(st.pt.shape, -1, np.int32)
    ids = st.rng.permutation(sum(need) + 2)
    at = 0
    for b, n in enumerate(need):
        out_pt[b, :n] = ids[at:at + n]
        at += n
    k, v = (torch.full((sum(need) + 2, page, hkv, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    binding.fp2_cache_expand(st.cache, st.dk, st.dv, st.dpt, torch.tensor(lens, dtype=torch.int32).cuda(), st.dks, st.dvs, k, v,
                             torch.from_numpy(out_pt).cuda(), st.ws)
    refs = [torch.full(k.shape, 9.0, dtype=torch.bfloat16) for _ in "kv"]
    for b, n in enumerate(lens):
        for ref, val in zip(refs, st.tokens(b)):
            for t in range(need[b]):
                ref[out_pt[b, t]] = 0.0
                rows = min(page, n - t * page)
                # (a product of e4m3 and fp32 has 28 bits: rounded to fp32 and then to BF16; the plain form alike)
                ref[out_pt[b, t], :rows] = val[t * page:t * page + rows].float().bfloat16()
    assert same(k, refs[0]) and same(v, refs[1])
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0
    if lens == [777]:
        bad = out_pt.copy()
        bad[0, 2] = sum(need) + 2
        binding.fp2_cache_expand(st.cache, st.dk, st.dv, st.dpt, torch.tensor(lens, dtype=torch.int32).cuda(), st.dks, st.dvs, k, v,
                                 torch.from_numpy(bad).cuda(), st.ws)
        code, words = binding.fp2_cache_read_status(st.cache, st.ws, raise_on_error=False)
        assert code == 1 and words[2] == 2 and same(k, refs[0])


def test_a_prompt_in_chunks_and_its_answer():
    """As an engine uses them, on an 8-bit cache with a scale per page: each chunk is appended, the sequence read back as BF16 pages
    and prefilled by the dense stage call; then tokens are decoded one by one and as a draft of three."""
    hq, hkv, page = 8, 2, 16
    chunks, steps = [(300, 130), (257, 400)], 6
    total = [sum(c[b] for c in chunks) for b in range(2)]
    st = Store(2, [0, 0], hq, hkv, page, seed=8, capacity=[n + 16 for n in total])
    rng = st.rng
    lens = [0, 0]
    k16, v16 = (torch.zeros(st.pool, page, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    for chunk in chunks:
        lens = [a + n for a, n in zip(lens, chunk)]
        n = sum(chunk)
        x = torch.from_numpy(rng.normal(0, 1, (n, 2 * hkv, D))).bfloat16().cuda()
        q = queries(rng, n, hq)
        run_append(st, x[:, :hkv], x[:, hkv:], lens, list(chunk))
        lk = torch.tensor(lens, dtype=torch.int32).cuda()
        binding.fp2_cache_expand(st.cache, st.dk, st.dv, st.dpt, lk, st.dks, st.dvs, k16, v16, st.dpt, st.ws)
        cu = [0, chunk[0], n]
        plan = binding.Plan(dict(num_seqs=2, total_q=n, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, block_size=128, tile_rows=128,
                                 page_size=page, num_pages=st.pool, max_pages_per_seq=st.mp, sink_tokens=256, window_tokens=512,
                                 use_correction=1, alpha=0.1, softmax_scale=0.0, dtype=0), cu, lens)
        out, lse = torch.empty(n, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, n, device="cuda")
        ws = plan.new_workspace()
        binding.fp2_dense_prefill(plan, q, k16, v16, st.dpt, torch.tensor(cu, dtype=torch.int32).cuda(), lk, None, None, None, out,
                                  lse, ws)
        binding.fp2_read_status(plan, ws)
        for b in range(2):
            k, v = st.tokens(b, lens[b])
            ro, rl, _, _ = attend(q[cu[b]:cu[b + 1]].cpu(), k, v, lens[b] - chunk[b], 0, 0)
            # the stage call's own tolerances (K and V are exact in BF16: powers of two times e4m3)
            assert float((out[cu[b]:cu[b + 1]].double().cpu() - ro).abs().max()) <= 2e-2
            assert float(((lse[:, cu[b]:cu[b + 1]].double().cpu() - rl).abs() / rl.abs().clamp_min(1.0)).max()) <= 1e-3
    for step in range(steps):
        n = 3 if step == steps - 1 else 1
        lens = [a + n for a in lens]
        x = torch.from_numpy(rng.normal(0, 2.0 ** (step % 3), (2 * n, 2 * hkv, D))).bfloat16().cuda()
        q = queries(rng, 2 * n, hq)
        run_append(st, x[:, :hkv], x[:, hkv:], lens, [n, n])
        for window, sinks in [(0, 0), (200, 4)]:
            out, lse = st.decode(q, [n, n], window, sinks, lens=lens)
            check(st, q, [n, n], out, lse, window, sinks, lens=lens)
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


@pytest.mark.parametrize("fmt", [0, 2])
def test_offsets_beyond_32_bits(fmt):
    """Pages at the far end of a pool of more than 2^32 bytes (and elements) per operand."""
    hkv, page = 8, 64
    pool = (2 ** 32) // (page * hkv * D) + 40
    cache = binding.Cache(dict(max_seqs=1, num_q_heads=8, num_kv_heads=hkv, head_dim=D, page_size=page, num_pages=pool,
                               max_pages_per_seq=4, format=fmt, softmax_scale=0.0))
    dt = torch.uint8 if fmt else torch.bfloat16
    k, v = (torch.empty(pool, page, hkv, D, dtype=dt, device="cuda") for _ in "kv")
    ks, vs = (torch.empty(pool, hkv, device="cuda") if fmt else None for _ in "kv")
    ids = [pool - 1, 3, pool - 30]
    pt = torch.tensor([ids + [-1]], dtype=torch.int32).cuda()
    x = torch.randn(150, 2 * hkv, D, device="cuda").bfloat16()
    cu, lk = torch.tensor([0, 150], dtype=torch.int32).cuda(), torch.tensor([150], dtype=torch.int32).cuda()
    ws = cache.new_workspace()
    binding.fp2_cache_append(cache, x[:, :hkv], x[:, hkv:], pt, cu, lk, k, v, ks, vs, ws)
    q = torch.randn(1, 8, D, device="cuda").bfloat16()
    out = torch.empty_like(q)
    binding.fp2_decode(cache, q, k, v, pt, torch.tensor([0, 1], dtype=torch.int32).cuda(), lk, ks, vs, out, None, ws)
    got = []
    for c, s in ((k, ks), (v, vs)):
        t = c[ids].cpu()
        t = t.view(E4M3).double() * s[ids].cpu().double()[:, None, :, None] if fmt else t.double()
        got.append(t.reshape(-1, hkv, D)[:150])
    for t, part in zip(got, (x[:, :hkv], x[:, hkv:])):
        assert float((t - part.double().cpu()).abs().max()) <= (float(part.abs().max()) * 2.0 ** -4 if fmt else 0.0)
    ro, _, mass, _ = attend(q.cpu(), got[0], got[1], 149, 0, 0)
    assert bool(((out.double().cpu() - ro).abs() <= 2.0 ** -8 * ro.abs() + 2.0 ** -9 * mass).all())
    assert binding.fp2_cache_read_status(cache, ws)[0] == 0


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("hq,hkv,page,lens,lq", [(64, 1, 16, [500, 77], [3, 1]), (40, 8, 8, [333], [2]), (5, 5, 32, [200, 3], [150, 3]),
                                                 (8, 2, 16, [700], [700])])
def test_decode_many_rows(fmt, hq, hkv, page, lens, lq):
    """More packed rows than one tile holds: wide groups, many queries, a whole prompt."""
    st = Store(fmt, lens, hq, hkv, page, seed=11)
    q = queries(st.rng, sum(lq), hq)
    for window, sinks in [(0, 0), (90, 20)]:
        out, lse = st.decode(q, lq, window, sinks)
        check(st, q, lq, out, lse, window, sinks)


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_sequences_that_share_a_prefix(fmt):
    """Two sequences with the same full pages in front: appending to each leaves these alone, both read them."""
    st = Store(fmt, [64, 64], 8, 2, 16, seed=12, capacity=[100, 100])
    st.pt[1, :4] = st.pt[0, :4]
    st.dpt = torch.from_numpy(st.pt).cuda()
    shared = st.dk[[int(p) for p in st.pt[0, :4]]].clone()
    x = torch.from_numpy(st.rng.normal(0, 3, (50, 4, D))).bfloat16().cuda()
    lens, news = [64 + 20, 64 + 30], [20, 30]
    run_append(st, x[:, :2], x[:, 2:], lens, news)
    assert same(st.dk[[int(p) for p in st.pt[0, :4]]], shared)
    q = queries(st.rng, 2, 8)
    out, lse = st.decode(q, [1, 1], lens=lens)
    check(st, q, [1, 1], out, lse, 0, 0, lens=lens)


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_local_layers_from_prompt_to_answer(fmt):
    """A layer with a sliding window: the prompt in two chunks through fp2_window_prefill, on the cache itself (BF16, per-head scales)
    or behind fp2_cache_expand (page scales), then tokens through fp2_decode with the same window and sinks."""
    hq, hkv, page, window, sinks = 8, 2, 16, 90, 5
    chunks, steps = [(200, 77), (150, 301)], 3
    total = [sum(c[b] for c in chunks) for b in range(2)]
    st = Store(fmt, [0, 0], hq, hkv, page, seed=21 + fmt, capacity=[n + 8 for n in total])
    rng, lens = st.rng, [0, 0]
    for chunk in chunks:
        lens = [a + n for a, n in zip(lens, chunk)]
        n = sum(chunk)
        x = torch.from_numpy(rng.normal(0, 1, (n, 2 * hkv, D))).bfloat16().cuda()
        q, q_scale = queries(rng, n, hq), None
        run_append(st, x[:, :hkv], x[:, hkv:], lens, list(chunk))
        lk = torch.tensor(lens, dtype=torch.int32).cuda()
        k, v, ks, vs = st.dk, st.dv, st.dks, st.dvs
        qv = q
        if fmt == 1:      # an FP8 plan takes e4m3 queries
            q_scale = torch.full((hq,), 1.0 / 64, device="cuda")
            qv = (q.float() * 64).clamp(-448, 448).to(E4M3).view(torch.uint8)
            q = qv.view(E4M3).float().cpu() / 64
        elif fmt == 2:
            k, v = (torch.zeros(st.pool, page, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
            binding.fp2_cache_expand(st.cache, st.dk, st.dv, st.dpt, lk, ks, vs, k, v, st.dpt, st.ws)
            ks = vs = None
        cu = [0, chunk[0], n]
        plan = binding.Plan(dict(num_seqs=2, total_q=n, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, block_size=128, tile_rows=128,
                                 page_size=page, num_pages=st.pool, max_pages_per_seq=st.mp, sink_tokens=256, window_tokens=512,
                                 use_correction=1, alpha=0.1, softmax_scale=0.0, dtype=1 if fmt == 1 else 0), cu, lens)
        out, lse = torch.empty(n, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(hq, n, device="cuda")
        ws = plan.new_workspace()
        binding.fp2_window_prefill(plan, qv, k, v, st.dpt, torch.tensor(cu, dtype=torch.int32).cuda(), lk, q_scale, ks, vs, window,
                                   sinks, out, lse, ws)
        binding.fp2_read_status(plan, ws)
        for b in range(2):
            kk, vv = st.tokens(b, lens[b])
            ro, rl, mass, _ = attend(q[cu[b]:cu[b + 1]].cpu(), kk, vv, lens[b] - chunk[b], window, sinks)
            # probabilities rounded to BF16 or F16 (2^-8 at most), logits and sums as in close() far below that, the output once
            err = (out[cu[b]:cu[b + 1]].double().cpu() - ro).abs()
            assert bool((err <= 2.0 ** -8 * ro.abs() + 1.1 * 2.0 ** -8 * mass).all())
            assert float((lse[:, cu[b]:cu[b + 1]].double().cpu() - rl).abs().max()) <= 1e-3
    for _ in range(steps):
        lens = [a + 1 for a in lens]
        x = torch.from_numpy(rng.normal(0, 1, (2, 2 * hkv, D))).bfloat16().cuda()
        q = queries(rng, 2, hq)
        run_append(st, x[:, :hkv], x[:, hkv:], lens, [1, 1])
        out, lse = st.decode(q, [1, 1], window, sinks, lens=lens)
        check(st, q, [1, 1], out, lse, window, sinks, lens=lens)
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


# ---------------------------------------------------------------------------------------------------------------------
# scales of pages at the ends of their range
# ---------------------------------------------------------------------------------------------------------------------
PAGE_SCALES = [
    # exponents of V's scales, page by page in turn; None: a page of zeros, at the writer's 2^-100
    [None, 36], [-120], [None], [120, None, -100], [-100, 36, 120, -60, 0], [60, -100],
]


def in_range(st, q, lq, out, window, sinks):
    """`out` with the exact value in the place of an infinity that stands for what BF16 cannot hold.  A code of 256 or more under a
    scale of 2^120 is 2^128 and up; the largest BF16 value is 255 2^120, and from 2^128 (1 - 2^-9) on the nearest is infinity.  The
    weights before that rounding are known to 2^-8 at best: a finite or infinite result is right from 2^128 (1 - 2^-7) on."""
    out, at = out.double().cpu(), 0
    for b, n in enumerate(lq):
        k, v = st.tokens(b)
        ro = attend(q[at:at + n].cpu(), k, v, st.lens[b] - n, window, sinks)[0]
        rows = out[at:at + n]
        beyond = torch.isinf(rows) & (ro.abs() >= 2.0 ** 128 * (1 - 2.0 ** -7)) & (torch.sign(ro) == torch.sign(rows))
        rows[beyond] = ro[beyond]
        at += n
    return out


@pytest.mark.parametrize("which", range(len(PAGE_SCALES)))
@pytest.mark.parametrize("sharp", [0.0, 1.0, 20.0])
@pytest.mark.parametrize("lens,lq", [([32], [1]), ([64, 300], [1, 5]), ([9000], [9])])
def test_decode_page_scales_far_apart(which, sharp, lens, lq):
    """The weights of pages of small values count like any others, and no sum leaves the range of 32 bits.  (Sharp queries: later
    tokens of small pages outweigh all earlier ones by far more than a sum's reference may lag.)"""
    st = Store(2, lens, 8, 2, 16, seed=which + 31)
    for b, n in enumerate(lens):
        for t in range(-(-n // 16)):
            e = PAGE_SCALES[which][t % len(PAGE_SCALES[which])]
            pid = int(st.pt[b, t])
            st.vs[pid] = 2.0 ** (-100 if e is None else e)
            if e is None:
                st.v[pid, :min(16, n - 16 * t)] = 0
    st.to_gpu()
    q = queries(st.rng, sum(lq), 8, sharp)
    for window, sinks in [(0, 0), (150, 20)]:
        out, lse = st.decode(q, lq, window, sinks)
        assert bool(torch.isfinite(lse).all())
        check(st, q, lq, in_range(st, q, lq, out, window, sinks), lse, window, sinks)
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


@pytest.mark.parametrize("exponent", [-100, -126, -140, 127])
def test_decode_a_million_tokens_of_equal_weight(exponent):
    """All logits are zero: lse = ln n, and out is V whatever its scale."""
    n, page = 1 << 20, 128
    cache = binding.Cache(dict(max_seqs=1, num_q_heads=1, num_kv_heads=1, head_dim=D, page_size=page, num_pages=n // page,
                               max_pages_per_seq=n // page, format=2, softmax_scale=0.0))
    k, v, ks, vs = cache.new_pages()
    vs.fill_(2.0 ** exponent)
    if exponent != -100:
        v.fill_(0x30)                      # 0.5
    pt = torch.randperm(n // page, device="cuda").to(torch.int32)[None].contiguous()
    cu, lk = torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    q = torch.randn(1, 1, D, device="cuda").bfloat16()
    out, lse, ws = torch.full_like(q, math.nan), torch.full((1, 1), math.nan, device="cuda"), cache.new_workspace()
    binding.fp2_decode(cache, q, k, v, pt, cu, lk, ks, vs, out, lse, ws)
    # n equal terms summed in 32 bits: by 2^-24 of the sum for every term of a lane's (n / 148 / 2 / 4 / 8 at least), and the joins
    assert abs(float(lse) - math.log(n)) <= 256 * 2.0 ** -24 + 2.0 ** -20
    want = 0.0 if exponent == -100 else 2.0 ** (exponent - 1)
    # the output's rounding, in steps of 2^-133 at the least, beside P's and the sums' as in close()
    assert bool(((out.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -15) * want + (2.0 ** -134 if want else 0.0)).all())


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("hkv,page", [(2, 16), (1, 128), (3, 8)])
@pytest.mark.parametrize("cu,lens", [
    ([0, 1000, 10, 20], [1000, 50, 15]),             # the second one falls; the others fit, the last one's rows are the first one's too
    ([0, 100, 50, 160], [300, 70, 115]),
    ([0, 700, 20, 700, 0, 700], [700, 30, 690, 5, 900]),        # more pages than the number of rows asks for
    ([0, 90, 5000, 30, 160], [100, 6000, 40, 130]),  # past the end of the rows
    ([0, 90, -7, 30, 160], [100, 20, 40, 135]),
    ([5, 40, 41, 41, 90, 3], [40, 700, 20, 60, 10]),
    ([0, 30, 60, 90], [30, 29, 40]),                 # ascending, but a sequence shorter than its new tokens
])
def test_append_leaves_out_the_sequence_that_does_not_fit_and_no_other(fmt, hkv, page, cu, lens):
    """Whatever stands in its neighbours' offsets, a sequence whose own fit is written, and written whole."""
    total = max(160, max(c for c in cu if c <= 1000))
    ok = [0 <= a <= b <= total and n >= b - a for a, b, n in zip(cu, cu[1:], lens)]
    news = [b - a if good else 0 for a, b, good in zip(cu, cu[1:], ok)]
    had = [n - new if good else 0 for n, new, good in zip(lens, news, ok)]
    st = Store(fmt, had, hkv, hkv, page, seed=17, capacity=[n if good else 64 for n, good in zip(lens, ok)])
    x = torch.from_numpy(st.rng.normal(0, 1, (total, 2 * hkv, D))).bfloat16().cuda()
    rows = torch.tensor([r for a, b, good in zip(cu, cu[1:], ok) if good for r in range(a, b)])
    want = plain_append(st, x[rows, :hkv], lens, news, "k") + plain_append(st, x[rows, hkv:], lens, news, "v")
    binding.fp2_cache_append(st.cache, x[:, :hkv], x[:, hkv:], st.dpt, torch.tensor(cu, dtype=torch.int32).cuda(),
                             torch.tensor(lens, dtype=torch.int32).cuda(), st.dk, st.dv, st.dks, st.dvs, st.ws)
    for got, ref in zip((st.dk, st.dks, st.dv, st.dvs), want):
        assert same(got, ref)
    code, words = binding.fp2_cache_read_status(st.cache, st.ws, raise_on_error=False)
    assert code == 1 and words[2] == 4


@pytest.mark.parametrize("fmt", [0, 2])
def test_more_sequences_than_one_search_step_tells_apart(fmt):
    """1500 sequences: appending, reading back, decoding (a search of 32 x 32 sequences, and scans of 128, take more than one round)."""
    rng = np.random.default_rng(51)
    news = [int(x) for x in rng.integers(0, 4, 1500)]
    had = [int(x) for x in rng.integers(0, 40, 1500)]
    lens = [a + n for a, n in zip(had, news)]
    st = Store(fmt, had, 2, 1, 16, seed=51, capacity=lens)
    x = torch.from_numpy(rng.normal(0, 1, (sum(news), 2, D))).bfloat16().cuda()
    want = plain_append(st, x[:, :1], lens, news, "k") + plain_append(st, x[:, 1:], lens, news, "v")
    run_append(st, x[:, :1], x[:, 1:], lens, news)
    for got, ref in zip((st.dk, st.dks, st.dv, st.dvs), want):
        assert same(got, ref)
    q = queries(rng, sum(news), 2)
    out, lse = st.decode(q, news, lens=lens)
    check(st, q, news, out, lse, 0, 0, lens=lens)
    if fmt:
        k, v = (torch.full((st.pool, 16, 1, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        binding.fp2_cache_expand(st.cache, st.dk, st.dv, st.dpt, torch.tensor(lens, dtype=torch.int32).cuda(), st.dks, st.dvs, k, v,
                                 st.dpt, st.ws)
        for o, i in ((k, 0), (v, 1)):
            got = o.cpu()
            for b, n in enumerate(lens):
                ref = torch.zeros(-(-n // 16) * 16, 1, D, dtype=torch.float64)
                ref[:n] = st.tokens(b, n)[i]
                assert torch.equal(got[[int(p) for p in st.pt[b, :-(-n // 16)]]].view(-1, 1, D).double(), ref)
    assert binding.fp2_cache_read_status(st.cache, st.ws)[0] == 0


def test_append_rounds_the_quotient_once():
    """Scales of the caller's that put quotients next to the middle between two e4m3 values: the code nearest to the exact quotient.
    (|x| against middle times scale: 29 bits, exact in 64.)"""
    rng = np.random.default_rng(4)
    hkv, n = 64, 16
    pos = e4m3_values()[:127].numpy()
    x = torch.from_numpy(rng.integers(128, 256, (n, hkv, D)) / 128 * np.where(rng.random((n, hkv, D)) < 0.5, -1, 1)).bfloat16()
    i = rng.integers(20, 100, hkv)
    middle = (pos[i] + pos[i + 1]) / 2
    s = (np.abs(x[0, :, 0].double().numpy()) / middle).astype(np.float32)      # token 0, dim 0 of every head is next to a tie
    s = np.nextafter(s, np.where(np.arange(hkv) % 3 == 0, 0, np.where(np.arange(hkv) % 3 == 1, np.inf, s)).astype(np.float32)).astype(np.float32)
    st = Store(1, [0], hkv, hkv, 16, capacity=[n])
    st.dks, st.dvs = torch.from_numpy(s).cuda(), torch.from_numpy(s).cuda()
    run_append(st, x.cuda(), x.cuda(), [n], [n])
    xd, sd = x.double().numpy(), s.astype(np.float64)[None, :, None]
    a = np.minimum(np.abs(xd), 448 * sd)
    # the last value whose product with the scale is not above |x|, found on the quotient and corrected by comparing products
    lo = np.clip(np.searchsorted(pos, a / sd, side="right") - 1, 0, 125)
    lo = np.where(pos[lo] * sd > a, lo - 1, lo)
    lo = np.where(pos[lo + 1] * sd <= a, np.minimum(lo + 1, 125), lo)
    border = (pos[lo] + pos[lo + 1]) / 2 * sd
    code = np.where((a > border) | ((a == border) & (lo % 2 == 1)), lo + 1, lo)
    code = torch.from_numpy((code + 128 * np.signbit(xd)).astype(np.uint8))
    got = st.dk[int(st.pt[0, 0])].cpu()
    assert torch.equal(got, code) and torch.equal(st.dv[int(st.pt[0, 0])].cpu(), code)


def nearest_bf16(x):
    """64-bit numbers to the nearest of eight significant bits, ties to even (normal numbers), as BF16."""
    m, e = np.frexp(x)
    return torch.from_numpy(np.ldexp(np.round(m * 256) / 256, e)).bfloat16()


def scales_at_ties():
    """fp32 scales under which a code lies next to the middle between two BF16 values: 1.625 * 1.5432693 among them."""
    rng = np.random.default_rng(3)
    code = np.arange(1, 2, 0.125)[rng.integers(0, 8, 500)]
    middle = (rng.integers(128, 256, 500) + 0.5) / 128
    s = (middle / code).astype(np.float32)
    s[0] = 1.5432693
    return np.nextafter(s, np.where(rng.random(500) < 0.5, 0, 9).astype(np.float32)).astype(np.float32)


@pytest.mark.parametrize("fmt", [1, 2])
def test_expand_rounds_once(fmt):
    """All codes under scales that put some of them next to a tie: the exact product (28 bits) rounded to BF16, and not to 32 bits on
    the way."""
    scales = torch.from_numpy(np.concatenate([scales_at_ties(), [np.float32(1.5432693)], np.float32(2.0) ** np.arange(-100, 100, 17)]).astype(np.float32))
    n = len(scales)
    hkv, pages = (n, 1) if fmt == 1 else (1, n)
    cache = binding.Cache(dict(max_seqs=1, num_q_heads=hkv, num_kv_heads=hkv, head_dim=D, page_size=8, num_pages=pages,
                               max_pages_per_seq=pages, format=fmt, softmax_scale=0.0))
    codes = torch.arange(256, dtype=torch.uint8).view(2, 1, D)          # tokens 0 and 1 of every page
    k = torch.zeros(pages, 8, hkv, D, dtype=torch.uint8)
    k[:, :2] = codes
    s = scales.cuda() if fmt == 1 else scales.cuda()[:, None].contiguous()
    pt = torch.arange(pages, dtype=torch.int32).cuda()[None].contiguous()
    out, o2 = (torch.zeros(pages, 8, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    binding.fp2_cache_expand(cache, k.cuda(), k.cuda(), pt, torch.tensor([8 * pages], dtype=torch.int32).cuda(), s, s, out, o2, pt,
                             cache.new_workspace())
    exact = codes.view(E4M3).double()[:, :, None, :] * scales.double()[None, None, :, None]       # [2, 1, n, D]
    finite = ~torch.isnan(exact)
    ref = nearest_bf16(torch.nan_to_num(exact).numpy())
    for got in (out, o2):
        got = got[:, :2].cpu()
        got = got.permute(1, 0, 2, 3) if fmt == 1 else got.permute(1, 2, 0, 3)
        assert bool(torch.isnan(got[~finite]).all()) and torch.equal(got[finite], ref[finite])


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("key,query", [(118, -124), (100, -100), (-100, 100), (-118, 110)])
def test_decode_small_queries_on_large_keys(fmt, key, query):
    """Logits of ordinary size from factors at the ends of their range."""
    st = Store(fmt, [200, 40], 8, 2, 16, seed=41)
    st.ks.fill_(2.0 ** (key - 6))          # codes are about 60
    st.to_gpu()
    q = torch.from_numpy(st.rng.normal(0, 1.5, (6, 8, D)) * 2.0 ** query).bfloat16().cuda()
    out, lse = st.decode(q, [5, 1])
    check(st, q, [5, 1], out, lse, 0, 0)


@pytest.mark.parametrize("page", [8, 16, 64])
def test_append_a_page_of_nothing_but_nan(page):
    """No finite magnitude in one head's page: the least scale, NaN codes; its neighbours as ever."""
    st = Store(2, [0], 2, 2, page, capacity=[3 * page])
    x = torch.from_numpy(st.rng.normal(0, 1, (3 * page, 2, D))).bfloat16()
    x[page:2 * page, 1] = math.nan
    x[2 * page:, 0] = math.nan
    x[2 * page, 0, 3] = math.inf              # and one with an infinity among them
    x = x.cuda()
    want = plain_append(st, x, [3 * page], [3 * page], "k")
    run_append(st, x, x, [3 * page], [3 * page])
    assert same(st.dk, want[0]) and same(st.dks, want[1]) and same(st.dv, want[0])
    one, two = int(st.pt[0, 1]), int(st.pt[0, 2])
    assert float(st.dks[one, 1]) == 2.0 ** -100 and float(st.dks[two, 0]) == 2.0 ** -100
    assert bool((st.dk[one, :, 1] & 0x7F == 0x7F).all()) and int(st.dk[two, 0, 0, 3]) == 0x7E


def test_append_rounds_what_a_page_holds_once():
    """A page under a caller's scale grows: its earlier tokens go to the e4m3 values nearest to code * scale / new scale, the product
    (28 bits) not rounded to 32 bits on the way."""
    rng = np.random.default_rng(6)
    hkv = 128
    pos = e4m3_values()[:127].numpy()
    code = np.arange(8, 16)[rng.integers(0, 8, hkv)] / 8.0                    # significands of the codes
    middle = (np.arange(8, 16)[rng.integers(0, 8, hkv)] + 0.5) / 8.0
    s = (middle / code).astype(np.float32)
    s = np.nextafter(s, np.where(np.arange(hkv) % 2 == 0, np.float32(0), np.float32(9))).astype(np.float32)
    st = Store(2, [5], hkv, hkv, 16, capacity=[6])
    pid = int(st.pt[0, 0])
    old = torch.from_numpy(rng.integers(0, 127, (5, hkv, D)).astype(np.uint8) + (128 * rng.integers(0, 2, (5, hkv, D))).astype(np.uint8))
    old[0] = torch.arange(D, dtype=torch.uint8)[None].clamp(max=126)          # every code
    for x, sc in ((st.dk, st.dks), (st.dv, st.dvs)):
        x[pid, :5] = old.cuda()
        sc[pid] = torch.from_numpy(s).cuda()
    new = torch.full((1, hkv, D), 448.0 * 4, dtype=torch.bfloat16, device="cuda")      # needs a scale of 4: s is below 2
    run_append(st, new, new, [6], [1])
    value = old.view(E4M3).double().numpy() * s.astype(np.float64)[None, :, None] / 4
    want = torch.from_numpy(nearest_e4m3(value))
    for x, sc in ((st.dk, st.dks), (st.dv, st.dvs)):
        assert torch.equal(x[pid, :5].cpu(), want) and bool((sc[pid] == 4.0).all()) and bool((x[pid, 5] == 0x7E).all())
