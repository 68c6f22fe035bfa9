"""What is timed next to the prefill calls of perf/cases.py: filling the paged KV cache, decoding from it, and local attention.

A case is one call of a serving engine on one attention layer, `op` says which:

  append  fp2_cache_append: keys and values of new tokens into their pages (quantised there where the cache holds 8 bits);
  decode  fp2_decode: attention of the newest few tokens of every sequence over its pages;
  expand  fp2_cache_expand: an 8-bit cache as BF16 pages, for the prefill calls;
  window  fp2_window_prefill: causal attention of a prompt (or a chunk of one) with a sliding window and sinks.

`fmt` is what the cache holds: "bf16", "head" (e4m3, one scale per KV head), "page" (e4m3, one scale per page and KV head).
Sequence b has a length between lo and hi (log-uniform, from `lens`), of which between nlo and nhi tokens are new.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
E4M3 = torch.float8_e4m3fn


def _case(op, fmt, seqs, lo, hi, nlo, nhi, hq, hkv, page, window=0, sinks=0, lens=0):
    return dict(op=op, fmt=fmt, seqs=seqs, lo=lo, hi=hi, nlo=nlo, nhi=nhi, hq=hq, hkv=hkv, page=page, window=window,
                sinks=sinks, lens=lens)


def listed():
    def named(name, *a, **k):
        return dict(_case(*a, **k), name=name)
    return [
        # one sequence decodes one token: the smallest call there is, latency alone
        named("append_one_token", "append", "page", 1, 777, 777, 1, 1, 32, 8, 16),
        # a full decode batch: a token each, most of them into pages that hold some already
        named("append_step_256", "append", "page", 256, 1, 600, 1, 1, 32, 8, 16, lens=1),
        # the prompts of a prefill step, behind prefixes that end inside a page
        named("append_prompts", "append", "page", 6, 3000, 15000, 2900, 14000, 32, 8, 64, lens=2),
        # a short prefix made readable for the prefill calls
        named("expand_short", "expand", "page", 1, 777, 777, 0, 0, 8, 2, 16),
        # the prefixes of a continuous batch
        named("expand_batch", "expand", "page", 16, 1024, 20000, 0, 0, 32, 8, 16, lens=3),
        # one short conversation
        named("decode_one_short", "decode", "bf16", 1, 777, 777, 1, 1, 32, 8, 16),
        # a decode batch of ragged lengths over 8-bit pages
        named("decode_batch_page", "decode", "page", 64, 200, 16384, 1, 1, 32, 8, 32, lens=4),
        # one long conversation, group size 7
        named("decode_128k_g7", "decode", "bf16", 1, 131072, 131072, 1, 1, 28, 4, 64),
        # drafted tokens verified with a window and sinks, 8 bits with a scale per head
        named("decode_draft_window", "decode", "head", 32, 500, 30000, 1, 5, 32, 8, 16, window=4096, sinks=4, lens=5),
        # a short prompt of a small model
        named("window_short", "window", "bf16", 1, 1000, 1000, 1000, 1000, 8, 2, 16, window=256, sinks=4),
        # a long prompt
        named("window_32k", "window", "bf16", 1, 32768, 32768, 32768, 32768, 32, 8, 64, window=4096, sinks=4),
        # chunks behind cached prefixes, 8 bits, group size 7
        named("window_chunks_fp8", "window", "head", 6, 1500, 40000, 700, 2048, 28, 4, 32, window=1000, sinks=130, lens=6),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "expand", "window"])
    hq, hkv = rng.choice([(32, 8), (28, 4), (8, 2), (4, 1), (14, 2), (8, 8), (40, 8)])
    page = rng.choice([8, 16, 32, 64, 128])
    lens = rng.randrange(1 << 20)
    if op == "append":
        fmt, seqs = rng.choice(["bf16", "head", "page", "page"]), _log_uniform(rng, 1, 200)
        nhi = 1 if rng.random() < 0.4 else _log_uniform(rng, 1, 40000 // seqs)
        return _case(op, fmt, seqs, 1, nhi + _log_uniform(rng, 1, 900), 1, nhi, hq, hkv, page, lens=lens)
    if op == "expand":
        fmt, seqs = rng.choice(["head", "page"]), _log_uniform(rng, 1, 40)
        hi = _log_uniform(rng, 40, 100000 // seqs)
        return _case(op, fmt, seqs, 1 + hi // 20, hi, 0, 0, hq, hkv, page, lens=lens)
    if op == "decode":
        fmt, seqs = rng.choice(["bf16", "head", "page", "page"]), _log_uniform(rng, 1, 96)
        hi = _log_uniform(rng, 30, 131072 // seqs if seqs < 8 else 16384)
        window, sinks = rng.choice([(0, 0), (_log_uniform(rng, 1, 8192), rng.choice([0, 4, 70]))])
        return _case(op, fmt, seqs, 1 + hi // 40, hi, 1, rng.choice([1, 1, 1, 2, 4, 7]), hq, hkv, page, window, sinks, lens)
    fmt, seqs = rng.choice(["bf16", "head"]), _log_uniform(rng, 1, 8)
    hi = _log_uniform(rng, 200, 32768 // seqs)
    return _case(op, fmt, seqs, 1 + hi // 4, hi, 1 + hi // 8, hi, hq, hkv, page, min(4096, _log_uniform(rng, 8, 4096)),
                 rng.choice([0, 4, 64, 300]), lens)


def _lengths(case):
    """[(tokens in the cache, new ones among them)] of every sequence."""
    rng = random.Random(case["lens"])
    out = []
    for _ in range(case["seqs"]):
        lk = _log_uniform(rng, case["lo"], case["hi"])
        out.append((lk, min(lk, _log_uniform(rng, case["nlo"], case["nhi"]) if case["nlo"] else 0)))
    return out


def _visible(case):
    """(visible (query, key) pairs, keys seen by some query) over all sequences."""
    w, s, pairs, keys = case["window"], case["sinks"], 0, 0
    for lk, n in _lengths(case):
        for p in ((lk - n, lk - 1) if n > 1 else (lk - 1,)):
            pairs += (n / (2 if n > 1 else 1)) * (p + 1 if not w or p < w else w + min(s, p + 1 - w))
        first = max(0, lk - n - w + 1) if w else 0
        keys += lk - first + min(s, first)
    return pairs, keys


def work(case):
    lens, hq, hkv = _lengths(case), case["hq"], case["hkv"]
    esz = 2 if case["fmt"] == "bf16" else 1
    new = sum(n for _, n in lens)
    if case["op"] == "append":
        return {"bytes": new * hkv * D * 2 * (2 + esz), "flops": new * hkv * D * 4}
    if case["op"] == "expand":
        n = sum(lk for lk, _ in lens) * hkv * D * 2
        return {"bytes": n * 3, "flops": n}
    pairs, keys = _visible(case)
    qsz = esz if case["op"] == "window" else 2
    return {"bytes": keys * hkv * D * 2 * esz + new * hq * (D * (2 + qsz) + 4), "flops": 4.0 * D * hq * pairs}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1000003 * seed + 17)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    lens, hq, hkv, p, fmt, op = _lengths(case), case["hq"], case["hkv"], case["page"], case["fmt"], case["op"]
    ns, new = len(lens), sum(n for _, n in lens)
    need = [-(-lk // p) for lk, _ in lens]
    pool, mp = sum(need) + 1, max(need)
    ids = torch.randperm(pool, generator=gen, device="cuda", dtype=torch.int64)[:sum(need)].to(torch.int32)
    host = torch.full((ns, mp), -1, dtype=torch.int64)
    at = 0
    for b, n in enumerate(need):
        host[b, :n] = torch.arange(at, at + n)
        at += n
    where = host.cuda()
    page_table = torch.where(where >= 0, ids[where.clamp_min(0)], torch.full_like(where, -1, dtype=torch.int32))
    s = dict(case=case, page_table=page_table.contiguous(), pool=pool, lens=lens,
             seqlens_k=torch.tensor([lk for lk, _ in lens], dtype=torch.int32).cuda(),
             cu=torch.tensor([0] + [n for _, n in lens], dtype=torch.int32).cumsum(0).to(torch.int32).cuda(), total=new,
             q_scale=None, k_scale=None, v_scale=None)
    # the cache: values about N(0, 1), keys with one loud channel in sixteen; 8 bits with the scales that their size asks for
    loud = 1.0 + 2.0 * (torch.arange(D, device="cuda") % 16 == 3).float()
    shape = (pool, p, hkv, D)
    if fmt == "bf16":
        s["k_cache"] = randn(*shape, dtype=torch.bfloat16).mul_(loud.bfloat16())
        s["v_cache"] = randn(*shape, dtype=torch.bfloat16)
    else:
        scales = []
        for name, amax in (("k", 13.0), ("v", 4.6)):
            if fmt == "head":
                scale = amax / 448 * torch.exp(0.3 * randn(hkv))
                each = torch.full((1, 1, hkv, 1), amax / 448, device="cuda")
            else:   # powers of two, those of quieter pages smaller
                e = torch.randint(-2, 1, (pool, hkv), generator=gen, device="cuda").float()
                scale = torch.exp2(e + math.ceil(math.log2(amax / 448)))
                each = torch.exp2(torch.full((1, 1, 1, 1), float(math.ceil(math.log2(amax / 448))), device="cuda"))
            x = randn(*shape, dtype=torch.bfloat16)
            if name == "k":
                x.mul_(loud.bfloat16())
            s[name + "_cache"] = (x / each.bfloat16()).clamp_(-448, 448).to(E4M3).view(torch.uint8)
            scales.append(scale.contiguous())
        s["k_scale"], s["v_scale"] = scales
    if op == "append":   # as slices of a fused projection's output; about every tenth token is loud
        fused = randn(new, 2 * hkv * D + hq * D, dtype=torch.bfloat16)
        fused *= torch.exp2(3.0 * (torch.rand(new, 1, generator=gen, device="cuda") < 0.1)).bfloat16()
        s["k_new"] = fused[:, hq * D:(hq + hkv) * D].view(new, hkv, D)
        s["v_new"] = fused[:, (hq + hkv) * D:].view(new, hkv, D)
        first = [max(0, lk - n) for lk, n in lens]
        s["seq_of"] = torch.tensor([b for b, (_, n) in enumerate(lens) for _ in range(n)]).cuda()
        s["pos_of"] = torch.tensor([f + i for f, (_, n) in zip(first, lens) for i in range(n)]).cuda()
        s["first"] = torch.tensor(first).cuda()
    elif op == "expand":
        s["out_page_table"] = where.to(torch.int32).contiguous()
        s["k_out"], s["v_out"] = (torch.zeros(sum(need), p, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        s["src_page"] = ids.long()
        s["rows_live"] = torch.cat([torch.full((n,), p) - torch.arange(n).eq(n - 1) * (n * p - lk)
                                    for n, (lk, _) in zip(need, lens)]).cuda()
    else:
        q = randn(new, hq, D, dtype=torch.bfloat16) * 1.2
        if op == "window" and fmt == "head":
            s["q_scale"] = 5.5 / 448 * torch.exp(0.3 * randn(hq))
            q = (q / (5.5 / 448)).clamp_(-448, 448).to(E4M3).view(torch.uint8)
        s["q"] = q
        s["out"] = torch.zeros(new, hq, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros(hq, new, dtype=torch.float32, device="cuda")
        # query blocks of one sequence each: (sequence, first query in it)
        c = max(n for _, n in lens) if op == "decode" else 512
        blocks = [(b, i) for b, (_, n) in enumerate(lens) for i in range(0, n, c)]
        s["block"] = c
        s["blk_seq"] = torch.tensor([b for b, _ in blocks]).cuda()
        s["blk_q0"] = torch.tensor([i for _, i in blocks]).cuda()
        number = {b: k for k, b in enumerate(blocks)}
        s["rows"] = torch.tensor([number[b, i - i % c] * c + i % c for b, (_, n) in enumerate(lens) for i in range(n)]).cuda()
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_2608_19758_b200 import binding
    c = s["case"]
    if c["op"] == "window":
        prm = dict(num_seqs=len(s["lens"]), total_q=s["total"], num_q_heads=c["hq"], num_kv_heads=c["hkv"], head_dim=D,
                   block_size=128, tile_rows=128, page_size=c["page"], num_pages=s["pool"],
                   max_pages_per_seq=s["page_table"].shape[1], sink_tokens=0, window_tokens=0, use_correction=0, alpha=0.1,
                   softmax_scale=0.0, dtype=0 if c["fmt"] == "bf16" else 1)
        s["plan"] = binding.Plan(prm, [0] + torch.tensor([n for _, n in s["lens"]]).cumsum(0).tolist(),
                                 [lk for lk, _ in s["lens"]])
        s["workspace"] = s["plan"].new_workspace()
        return
    prm = dict(max_seqs=len(s["lens"]), num_q_heads=c["hq"], num_kv_heads=c["hkv"], head_dim=D, page_size=c["page"],
               num_pages=s["pool"], max_pages_per_seq=s["page_table"].shape[1], softmax_scale=0.0,
               format={"bf16": 0, "head": 1, "page": 2}[c["fmt"]])
    s["cache"] = binding.Cache(prm)
    s["workspace"] = s["cache"].new_workspace()


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "append":
        return _append(s)
    if op == "expand":
        return _expand(s)
    return _attend(s)


def _values(s, x):
    return x.view(E4M3) if s["case"]["fmt"] != "bf16" else x


def _run_own(s):
    from paper_2608_19758_b200 import binding
    c = s["case"]
    if c["op"] == "append":
        binding.fp2_cache_append(s["cache"], s["k_new"], s["v_new"], s["page_table"], s["cu"], s["seqlens_k"], s["k_cache"],
                                 s["v_cache"], s["k_scale"], s["v_scale"], s["workspace"])
        return _values(s, s["k_cache"]), _values(s, s["v_cache"]), s["k_scale"], s["v_scale"]
    if c["op"] == "expand":
        binding.fp2_cache_expand(s["cache"], s["k_cache"], s["v_cache"], s["page_table"], s["seqlens_k"], s["k_scale"],
                                 s["v_scale"], s["k_out"], s["v_out"], s["out_page_table"], s["workspace"])
        return s["k_out"], s["v_out"]
    if c["op"] == "decode":
        binding.fp2_decode(s["cache"], s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["cu"], s["seqlens_k"],
                           s["k_scale"], s["v_scale"], s["out"], s["lse"], s["workspace"], window_tokens=c["window"],
                           sink_tokens=c["sinks"])
        return s["out"], s["lse"]
    binding.fp2_window_prefill(s["plan"], s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["cu"], s["seqlens_k"],
                               s["q_scale"], s["k_scale"], s["v_scale"], c["window"], c["sinks"], s["out"], s["lse"],
                               s["workspace"])
    return s["out"], s["lse"]


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _append(s):
    c = s["case"]
    p, hkv, fmt = c["page"], c["hkv"], c["fmt"]
    page = s["page_table"][s["seq_of"], s["pos_of"] // p].long()
    row = s["pos_of"] % p
    # the page that each sequence's new tokens begin in, and whether a row of it was there before
    live = s["first"] < s["seqlens_k"]
    begin = s["page_table"].gather(1, (s["first"] // p).clamp_max(s["page_table"].shape[1] - 1)[:, None])[:, 0].long()
    begin = torch.where(live, begin, torch.zeros_like(begin))
    kept = (torch.arange(p, device="cuda")[None] < (s["first"] % p)[:, None]) & live[:, None]     # [seqs, p]
    old = kept.any(1)
    for x, cache, scale in ((s["k_new"], s["k_cache"], s["k_scale"]), (s["v_new"], s["v_cache"], s["v_scale"])):
        if fmt == "bf16":
            cache[page, row] = x
            continue
        codes = cache.view(E4M3)
        x = x.float()
        if fmt == "head":
            codes.view(torch.uint8)[page, row] = (x / scale[:, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
            continue
        amax = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax", include_self=True)
        f, e = torch.frexp(amax)
        want = torch.ldexp(torch.ones_like(f), torch.where(f > 0.875, e - 8, e - 9))
        want = torch.where(amax > 0, want, torch.zeros_like(want)).clamp_min(2.0 ** -100)
        before = torch.where(old[:, None], scale[begin], torch.zeros_like(scale[begin]))            # [seqs, hkv]
        had = torch.zeros_like(scale).index_reduce_(0, begin, before, "amax", include_self=True)
        now = torch.maximum(want, had)
        back = codes[begin].float() * before[:, None, :, None]
        back = (back / now[begin][:, None, :, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        back = torch.where(kept[:, :, None, None], back, cache[begin])
        cache.index_copy_(0, begin, back)
        cache[page, row] = (x / now[page][:, :, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        scale.index_copy_(0, page, now[page])
    return _values(s, s["k_cache"]), _values(s, s["v_cache"]), s["k_scale"], s["v_scale"]


def _scaled(s, codes, scale, page):
    """Values of gathered cache rows [..., hkv, D]; `page`: their pages [...]."""
    if s["case"]["fmt"] == "bf16":
        return codes.float()
    x = codes.view(E4M3).float()
    return x.mul_((scale[page] if s["case"]["fmt"] == "page" else scale)[..., None])


def _expand(s):
    p = s["case"]["page"]
    live = torch.arange(p, device="cuda")[None] < s["rows_live"][:, None]
    for cache, scale, out in ((s["k_cache"], s["k_scale"], s["k_out"]), (s["v_cache"], s["v_scale"], s["v_out"])):
        page = s["src_page"][:, None].expand(-1, p)
        x = _scaled(s, cache[s["src_page"]], scale, page)
        out.copy_(torch.where(live[:, :, None, None], x, torch.zeros_like(x)))
    return s["k_out"], s["v_out"]


def _attend(s):
    c = s["case"]
    hq, hkv, p, w, sinks, n = c["hq"], c["hkv"], c["page"], c["window"], c["sinks"], s["block"]
    g, dev = hq // hkv, "cuda"
    lk = s["seqlens_k"].long()[s["blk_seq"]]
    lq = (s["cu"][1:] - s["cu"][:-1]).long()[s["blk_seq"]]
    i = s["blk_q0"][:, None] + torch.arange(n, device=dev)[None]                       # [blk, n]
    pos = (lk - lq)[:, None] + i
    rows = (s["cu"].long()[s["blk_seq"]][:, None] + i).clamp_max(max(s["total"] - 1, 0))
    # keys of a block: the span of its windows, then the sinks in front of it
    begin = pos[:, 0] - w + 1 if w else torch.zeros_like(lk)
    span = w + n - 1 if w else max(a for a, _ in s["lens"])
    j = begin[:, None] + torch.arange(span, device=dev)[None]
    front = torch.arange(sinks if w else 0, device=dev)[None].expand(len(lk), -1)
    inside = torch.cat([(j >= 0) & (j < lk[:, None]), (front < begin[:, None]) & (front < lk[:, None])], 1)
    j = torch.cat([j, front], 1)
    j0 = torch.where(inside, j, torch.zeros_like(j))
    page = s["page_table"][s["blk_seq"][:, None], j0 // p].long()
    slot = page * p + j0 % p
    k = _scaled(s, s["k_cache"].view(-1, hkv, D)[slot], s["k_scale"], page)            # [blk, T, hkv, D]
    v = _scaled(s, s["v_cache"].view(-1, hkv, D)[slot], s["v_scale"], page)
    q = s["q"][rows]
    q = q.view(E4M3).float() * s["q_scale"][:, None] if s["q_scale"] is not None else q.float()
    q = q.view(-1, n, hkv, g, D).permute(0, 2, 3, 1, 4).reshape(-1, hkv, g * n, D)      # head-major, then query
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(1.0 / math.sqrt(D))                 # [blk, hkv, g n, T]
    see = inside[:, None] & (j[:, None] <= pos[:, :, None])
    if w:
        see &= (pos[:, :, None] - j[:, None] < w) | (j[:, None] < sinks)
    see = see[:, None, None].expand(-1, 1, g, -1, -1).reshape(len(lk), 1, g * n, -1)
    x.masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-1e30)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x, v.permute(0, 2, 1, 3)) / total
    lse = m + torch.log(total)
    o = o.view(-1, hkv, g, n, D).permute(0, 3, 1, 2, 4).reshape(-1, hq, D)
    lse = lse.view(-1, hkv, g, n).permute(0, 3, 1, 2).reshape(-1, hq)
    s["out"].copy_(o[s["rows"]])
    s["lse"].copy_(lse[s["rows"]].T)
    return s["out"], s["lse"]


# ---------------------------------------------------------------------------------------------------------------------
# the operators' definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _nearest_e4m3(x):
    """The value of e4m3 (1 - 4 - 3 bits, largest 448, steps of 2^-9 below 2^-6) nearest to x, ties to even; saturating."""
    _, e = torch.frexp(x.abs())
    step = torch.exp2((e.double() - 1).clamp(-6, 8) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _pages_of(s, b, lk):
    p = s["case"]["page"]
    return s["page_table"][b, :-(-lk // p)].long()


def _tokens(s, b, lk, name):
    """Keys or values of sequence b as [tokens, hkv, D] in 64 bits."""
    fmt, pages = s["case"]["fmt"], _pages_of(s, b, lk)
    x = s[name + "_cache"][pages]
    if fmt == "bf16":
        x = x.double()
    else:
        scale = s[name + "_scale"].double()
        x = x.view(E4M3).double() * (scale[None, None, :, None] if fmt == "head" else scale[pages][:, None, :, None])
    return x.reshape(-1, s["case"]["hkv"], D)[:lk]


def exact(case, seed):
    s = prepare(case, seed)
    p, hq, hkv = case["page"], case["hq"], case["hkv"]
    if case["op"] == "append":
        return _exact_append(s)
    if case["op"] == "expand":
        out = [torch.zeros(s["k_out"].shape, dtype=torch.float64, device="cuda") for _ in "kv"]
        at = 0
        for b, (lk, _) in enumerate(s["lens"]):
            for o, name in zip(out, "kv"):
                o.view(-1, hkv, D)[at * p:at * p + lk] = _tokens(s, b, lk, name)
            at += -(-lk // p)
        return tuple(out)
    out = torch.zeros(s["total"], hq, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(hq, s["total"], dtype=torch.float64, device="cuda")
    at = 0
    for b, (lk, n) in enumerate(s["lens"]):
        if not n:
            continue
        k, v = _tokens(s, b, lk, "k"), _tokens(s, b, lk, "v")
        pos = torch.arange(lk - n, lk, device="cuda")[:, None]
        key = torch.arange(lk, device="cuda")[None]
        hidden = key > pos
        if case["window"]:
            hidden |= (key <= pos - case["window"]) & (key >= case["sinks"])
        for h in range(hq):
            q = s["q"][at:at + n, h]
            q = q.view(E4M3).double() * s["q_scale"][h].double() if s["q_scale"] is not None else q.double()
            x = (q @ k[:, h // (hq // hkv)].T) / math.sqrt(D)
            x[hidden] = -math.inf
            lse[h, at:at + n] = torch.logsumexp(x, 1)
            out[at:at + n, h] = torch.softmax(x, 1) @ v[:, h // (hq // hkv)]
        at += n
    return out, lse


def _exact_append(s):
    case = s["case"]
    p, fmt = case["page"], case["fmt"]
    got = []
    for name in "kv":
        new, cache = s[name + "_new"].double(), s[name + "_cache"]
        scale = None if fmt == "bf16" else s[name + "_scale"].double()
        values = cache.double() if fmt == "bf16" else cache.view(E4M3).double()
        at = 0
        for b, (lk, n) in enumerate(s["lens"]):
            pages, first = _pages_of(s, b, lk), lk - n
            x, at = new[at:at + n], at + n
            if fmt != "page":
                place = pages[torch.arange(first, lk, device="cuda") // p] * p + torch.arange(first, lk, device="cuda") % p
                values.view(-1, *values.shape[2:])[place] = x if fmt == "bf16" else _nearest_e4m3(x / scale[:, None])
                continue
            for t in range(first // p, -(-lk // p)):
                page, lo, hi = pages[t], max(first, t * p), min(lk, (t + 1) * p)
                most = x[lo - first:hi - first].abs().amax((0, 2))
                size = torch.exp2(torch.ceil(torch.log2(most / 448))).clamp_min(2.0 ** -100)
                if lo > t * p:
                    held = torch.maximum(size, scale[page])
                    values[page, :lo - t * p] = _nearest_e4m3(values[page, :lo - t * p] * (scale[page] / held)[:, None])
                    size = held
                scale[page] = size
                values[page, lo - t * p:hi - t * p] = _nearest_e4m3(x[lo - first:hi - first] / size[:, None])
        got += [values, scale]
    return got[0], got[2], got[1], got[3]
