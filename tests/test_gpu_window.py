"""fp2_window_prefill: local attention of prompts and chunks against a plain form in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2608_19758_b200 import binding

pytestmark = pytest.mark.gpu
D = 128
E4M3 = torch.float8_e4m3fn
NAN8 = 0x7F


class Prompt:
    """Sequences (tokens in the cache, new ones among them); rows of last pages behind a sequence and spare pages hold NaN."""

    def __init__(self, fp8, seqs, hq, hkv, page, seed=0, sharp=1.5):
        self.fp8, self.seqs, self.hq, self.hkv, self.page = fp8, seqs, hq, hkv, page
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        need = [-(-lk // page) for lk, _ in seqs]
        self.pool, mp = sum(need) + 2, max(max(need), 1)
        ids = np.random.default_rng(seed).permutation(self.pool)
        self.pt, at = np.full((len(seqs), mp), -1, np.int32), 0
        for b, n in enumerate(need):
            self.pt[b, :n] = ids[at:at + n]
            at += n
        total = sum(n for _, n in seqs)
        shape = (self.pool, page, hkv, D)
        q = randn(total, hq, D) * sharp
        self.qs = self.ks = self.vs = None
        if fp8:
            self.q = (q * 60).clamp(-448, 448).to(E4M3).view(torch.uint8)
            self.k, self.v = (torch.full(shape, NAN8, dtype=torch.uint8, device="cuda") for _ in "kv")
            self.qs, self.ks, self.vs = (torch.exp(0.3 * randn(n)) / 60 for n in (hq, hkv, hkv))
        else:
            self.q = q.bfloat16()
            self.k, self.v = (torch.full(shape, math.nan, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        for b, (lk, _) in enumerate(seqs):
            for t in range(need[b]):
                rows = min(page, lk - t * page)
                for x in (self.k, self.v):
                    val = randn(rows, hkv, D)
                    x[int(self.pt[b, t]), :rows] = (val * 60).clamp(-448, 448).to(E4M3).view(torch.uint8) if fp8 else val.bfloat16()
        self.cu = np.concatenate([[0], np.cumsum([n for _, n in seqs])]).astype(np.int32)
        self.plan = binding.Plan(dict(num_seqs=len(seqs), total_q=total, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                                      block_size=128, tile_rows=128, page_size=page, num_pages=self.pool, max_pages_per_seq=mp,
                                      sink_tokens=256, window_tokens=512, use_correction=1, alpha=0.1, softmax_scale=0.0,
                                      dtype=1 if fp8 else 0), self.cu.tolist(), [lk for lk, _ in seqs])
        self.ws = self.plan.new_workspace()
        self.dpt = torch.from_numpy(self.pt).cuda()
        self.dcu = torch.from_numpy(self.cu).cuda()
        self.lk = torch.tensor([lk for lk, _ in seqs], dtype=torch.int32).cuda()

    def run(self, window, sinks, lse=True, stream=None, ws=None):
        out = torch.full((int(self.cu[-1]), self.hq, D), math.nan, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.hq, out.shape[0]), math.nan, device="cuda") if lse else None
        binding.fp2_window_prefill(self.plan, self.q, self.k, self.v, self.dpt, self.dcu, self.lk, self.qs, self.ks, self.vs, window,
                                   sinks, out, lse, self.ws if ws is None else ws, stream=stream)
        return out, lse

    def values(self, x, scale):
        return x.view(E4M3).double() * scale.double()[:, None] if self.fp8 else x.double()

    def check(self, out, lse, window, sinks):
        """Tolerances.  Logits: d = 2^-17 of sum |q k| scale (128 products summed in fp32, 128 * 2^-24) + 2^-20 (scaling, exponential,
        logarithm), sums of n positive terms n 2^-24.  Probabilities are rounded to BF16 (2^-8) or F16 (2^-11, and 2^-25 of the
        largest where that runs out); the output once: 2^-8."""
        g = self.hq // self.hkv
        for b, (lk, n) in enumerate(self.seqs):
            if not n:
                continue
            slot = torch.from_numpy(self.pt[b, np.arange(lk) // self.page].astype(np.int64) * self.page + np.arange(lk) % self.page).cuda()
            rows = slice(int(self.cu[b]), int(self.cu[b + 1]))
            pos, key = torch.arange(lk - n, lk, device="cuda")[:, None], torch.arange(lk, device="cuda")[None]
            hidden = (key > pos) | ((pos - key >= window) & (key >= sinks))
            used = ~hidden.all(0)
            for h in range(self.hq):
                q = self.values(self.q[rows], self.qs)[:, h]
                k, v = (torch.where(used[:, None], self.values(x.view(-1, self.hkv, D)[slot], s)[:, h // g], torch.zeros((), dtype=torch.float64, device="cuda"))
                        for x, s in ((self.k, self.ks), (self.v, self.vs)))
                x = (q @ k.T) / math.sqrt(D)
                size = float((q.abs() @ k.abs().T).max()) / math.sqrt(D)
                x[hidden] = -math.inf
                want_l = torch.logsumexp(x, 1)
                w = torch.exp(x - want_l[:, None])
                want, mass = w @ v, w @ v.abs()
                d = 2.0 ** -17 * size + 2.0 ** -20 + lk * 2.0 ** -24
                p = 2.0 ** -11 if self.fp8 else 2.0 ** -8
                tol = 2.0 ** -8 * want.abs() + (2 * d + p) * (1 + 2.0 ** -8) * mass + (2.0 ** -25 * lk * float(v.abs().max()) if self.fp8 else 0.0)
                err = (out[rows, h].double() - want).abs()
                assert bool((err <= tol).all()), (b, h, float((err - tol).max()), float(err.max()))
                if lse is not None:
                    err = (lse[h, rows].double() - want_l).abs()
                    assert bool((err <= d + 2.0 ** -22 * want_l.abs()).all()), (b, h, float(err.max()))


SEQS = [[(1, 1)], [(777, 777)], [(300, 300), (0, 0), (129, 1), (1000, 37), (128, 128), (700, 0)], [(1500, 513)]]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,page", [((8, 2), 16), ((4, 1), 128), ((14, 2), 64), ((4, 4), 8), ((6, 2), 32), ((12, 1), 16)])
@pytest.mark.parametrize("which", range(len(SEQS)))
def test_window(fp8, heads, page, which):
    p = Prompt(fp8, SEQS[which], *heads, page, seed=which)
    for window, sinks in [(1, 0), (5, 3), (100, 4), (128, 128), (129, 300), (400, 0), (1 << 30, 5), (2 ** 31 - 1, 2 ** 31 - 1)]:
        out, lse = p.run(window, sinks)
        p.check(out, lse, window, sinks)
    code, words = binding.fp2_read_status(p.plan, p.ws)
    assert code == 0 and p.plan.last_launch_count() == 2


@pytest.mark.parametrize("fp8", [False, True])
def test_window_longer(fp8):
    """Many units per worker; FP8: long enough for V as F16 to be laid out once."""
    p = Prompt(fp8, [(6000, 6000), (2500, 900)], 28, 4, 32, seed=3)
    for window, sinks in [(1000, 4), (700, 130)]:
        out, lse = p.run(window, sinks)
        p.check(out, lse, window, sinks)
        o2, l2 = p.run(window, sinks)
        assert torch.equal(out.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, l2)
    o2, _ = p.run(700, 130, lse=False)
    assert torch.equal(out.view(torch.int16), o2.view(torch.int16))
    binding.fp2_read_status(p.plan, p.ws)


def test_window_as_wide_as_the_sequence_is_dense_attention():
    for fp8 in (False, True):
        p = Prompt(fp8, [(640, 640), (1024, 256)], 8, 2, 64, seed=5)      # (full last blocks: what fp2_dense_prefill asks for)
        out, lse = p.run(4096, 0)
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        binding.fp2_dense_prefill(p.plan, p.q, p.k, p.v, p.dpt, p.dcu, p.lk, p.qs, p.ks, p.vs, o2, l2, p.ws)
        p.check(o2, l2, 4096, 0)
        p.check(out, lse, 4096, 0)


@pytest.mark.parametrize("fp8,tokens", [(False, 900), (True, 900), (True, 7000)])
def test_window_hidden_places_do_not_matter(fp8, tokens):
    """A chunk behind a long prefix: pages in front of its windows are gone, tokens there hold NaN."""
    hq, hkv = (28, 4) if tokens > 1000 else (8, 2)
    p = Prompt(fp8, [(tokens, tokens - 600)], hq, hkv, 16, seed=6)
    window, sinks = 130, 20
    clean, clean_l = p.run(window, sinks)
    p.check(clean, clean_l, window, sinks)
    first = 600 - window + 1                       # first token of the first window
    for tok in range(sinks, first):
        for x in (p.k, p.v):
            x.view(-1, hkv, D)[int(p.pt[0, tok // 16]) * 16 + tok % 16] = NAN8 if fp8 else (math.nan if tok % 3 else math.inf)
    for t in range(2, first // 16):
        p.dpt[0, t] = -1 if t % 2 else p.pool + 3
    out, lse = p.run(window, sinks)
    assert torch.equal(out.view(torch.int16), clean.view(torch.int16)) and torch.equal(lse, clean_l)
    code, words = binding.fp2_read_status(p.plan, p.ws, raise_on_error=False)
    assert code == 0 and not any(words)
    # a page that some query sees: reported
    p.dpt[0, first // 16 + 1] = -1
    p.run(window, sinks)
    code, words = binding.fp2_read_status(p.plan, p.ws, raise_on_error=False)
    assert code == 1 and words[2] == 2 and words[0] == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_window_next_to_the_other_stage_calls_on_one_workspace(fp8):
    """Local and global layers of one model: the calls share plan and workspace; captured and replayed, on a side stream too."""
    p = Prompt(fp8, [(1300, 1300), (800, 300)], 8, 2, 16, seed=7)
    for x in (p.k, p.v):     # (what the other calls ask for behind the sequences' ends)
        x[x.view(torch.int8 if fp8 else torch.int16) == (NAN8 if fp8 else torch.full((1,), math.nan, dtype=torch.bfloat16).view(torch.int16).item())] = 0
    ref, ref_l = p.run(200, 4)
    p.check(ref, ref_l, 200, 4)
    dense, dense_l = torch.empty_like(ref), torch.empty_like(ref_l)

    def layer(o, l):
        binding.fp2_dense_prefill(p.plan, p.q, p.k, p.v, p.dpt, p.dcu, p.lk, p.qs, p.ks, p.vs, dense, dense_l, p.ws)
        binding.fp2_window_prefill(p.plan, p.q, p.k, p.v, p.dpt, p.dcu, p.lk, p.qs, p.ks, p.vs, 200, 4, o, l, p.ws)

    for _ in range(3):
        o, l = torch.full_like(ref, math.nan), torch.full_like(ref_l, math.nan)
        layer(o, l)
        assert torch.equal(o.view(torch.int16), ref.view(torch.int16)) and torch.equal(l, ref_l)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(o, l)
    for _ in range(3):
        o.fill_(math.nan)
        dense.fill_(math.nan)
        graph.replay()
        assert torch.equal(o.view(torch.int16), ref.view(torch.int16))
        p.check(dense, dense_l, 1 << 20, 0)
    side, ws = torch.cuda.Stream(), p.plan.new_workspace()
    torch.cuda.synchronize()
    o, l = p.run(200, 4, stream=side, ws=ws)
    side.synchronize()
    assert torch.equal(o.view(torch.int16), ref.view(torch.int16)) and torch.equal(l, ref_l)
    binding.fp2_read_status(p.plan, p.ws)
    binding.fp2_read_status(p.plan, ws)


@pytest.mark.parametrize("fp8", [False, True])
def test_window_tokens_behind_a_tile_do_not_matter(fp8):
    """The newest tokens hold NaN: the queries that see them get NaN, those of earlier 128-row tiles (32 queries here) are as before."""
    p = Prompt(fp8, [(600, 600)], 8, 2, 16, seed=13)
    clean, clean_l = p.run(100, 4)
    for tok in (590, 599):
        for x in (p.k, p.v):
            x.view(-1, 2, D)[int(p.pt[0, tok // 16]) * 16 + tok % 16] = NAN8 if fp8 else math.nan
    out, lse = p.run(100, 4)
    assert torch.equal(out[:576].view(torch.int16), clean[:576].view(torch.int16)) and torch.equal(lse[:, :576], clean_l[:, :576])
    assert bool(torch.isnan(out[590:].float()).all()) and bool(torch.isnan(lse[:, 590:]).all())
    binding.fp2_read_status(p.plan, p.ws)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_window_on_the_oracles_inputs(dtype):
    """The generator's inputs (locality, sinks, vertical keys) through the helper of the other stage calls, against the oracle's dense
    path where the window covers everything."""
    from oracle import fp2_oracle as O
    from paper_2608_19758_b200 import inputs
    spec = inputs.small_spec(seqs=[(700, 100), (300, 0)], num_q_heads=8, num_kv_heads=2, page_size=16, config_id=97, dtype=dtype)
    case = inputs.make_case(spec)
    dc = binding.DeviceCase(case)
    dc.poison = True
    dc.window(1 << 20)
    dc.status()
    wl = O.Workload(O.Params.from_dict(case.params()), **inputs.oracle_args(case))
    ref, lref = O.scatter_output(wl, O.oracle_attend(wl, None, dense=True), case.total_q)
    assert np.abs(dc.out.float().cpu().numpy() - ref).max() <= (2e-2 if dtype == "bf16" else 6e-2)     # the stage calls' tolerances
    assert (np.abs(dc.lse.cpu().numpy() - lref) / np.maximum(np.abs(lref), 1)).max() <= 1e-3
