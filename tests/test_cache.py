"""The paged KV cache on the host: what its calls refuse, before anything is launched."""
import ctypes as C
import types

import pytest
import torch

from paper_2608_19758_b200 import binding


def cache_params(**kw):
    p = dict(max_seqs=4, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, num_pages=64, max_pages_per_seq=32,
             format=2, softmax_scale=0.0)
    p.update(kw)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=64), 2), (dict(page_size=48), 2), (dict(page_size=4), 2), (dict(page_size=256), 2), (dict(page_size=0), 2),
    (dict(format=3), 2), (dict(format=-1), 2), (dict(num_q_heads=7), 1), (dict(num_q_heads=0), 1), (dict(num_kv_heads=0), 1),
    (dict(max_seqs=0), 1), (dict(num_pages=0), 1), (dict(max_pages_per_seq=0), 1), (dict(softmax_scale=-1.0), 1),
    (dict(softmax_scale=float("nan")), 1), (dict(softmax_scale=float("inf")), 1), (dict(max_pages_per_seq=(1 << 26) + 1), 3),
    (dict(num_q_heads=1 << 14, num_kv_heads=1 << 14), 3),
])
def test_cache_create_refuses(kw, code):
    with pytest.raises(binding.Fp2Error) as e:
        binding.Cache(cache_params(**kw))
    assert e.value.code == code


def test_null_handles_and_pointers():
    lib = binding.load()
    assert lib.fp2_cache_create(None, None) == 1
    assert lib.fp2_cache_sizes(None, None) == 1
    lib.fp2_cache_destroy(None)
    p = C.c_void_p(4096)
    assert lib.fp2_cache_append(None, p, p, 256, p, p, p, 1, 1, p, p, p, p, p, None) == 1
    assert lib.fp2_cache_expand(None, p, p, p, p, 1, p, p, p, p, p, 1, p, None) == 1
    assert lib.fp2_decode(None, p, 1024, p, p, p, p, p, 1, 1, p, p, 0, 0, p, None, p, None) == 1
    assert lib.fp2_cache_read_status(None, p, None, None) == 1


def _append(lib, h, **kw):
    a = dict(k_new=4096, v_new=4096, stride=256, pt=4096, cu=4096, lk=4096, ns=2, total=3, k=4096, v=4096, ks=4096, vs=4096, ws=4096)
    a.update(kw)
    return lib.fp2_cache_append(h, a["k_new"], a["v_new"], a["stride"], a["pt"], a["cu"], a["lk"], a["ns"], a["total"], a["k"],
                                a["v"], a["ks"], a["vs"], a["ws"], None)


def _expand(lib, h, **kw):
    a = dict(k=4096, v=4096, pt=4096, lk=4096, ns=2, ks=4096, vs=4096, ko=4096, vo=4096, opt=4096, pages=8, ws=4096)
    a.update(kw)
    return lib.fp2_cache_expand(h, a["k"], a["v"], a["pt"], a["lk"], a["ns"], a["ks"], a["vs"], a["ko"], a["vo"], a["opt"],
                                a["pages"], a["ws"], None)


def _decode(lib, h, **kw):
    a = dict(q=4096, stride=1024, k=4096, v=4096, pt=4096, cu=4096, lk=4096, ns=2, total=3, ks=4096, vs=4096, w=0, s=0, out=4096,
             lse=None, ws=4096)
    a.update(kw)
    return lib.fp2_decode(h, a["q"], a["stride"], a["k"], a["v"], a["pt"], a["cu"], a["lk"], a["ns"], a["total"], a["ks"],
                          a["vs"], a["w"], a["s"], a["out"], a["lse"], a["ws"], None)


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_calls_refuse_bad_arguments_before_they_look_for_a_device(fmt):
    """(Made-up addresses: only where there is no device, so that the good call ends with FP2_ERR_CUDA.)"""
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    lib = binding.load()
    cache = binding.Cache(cache_params(format=fmt))
    h = cache.handle
    common = [dict(k=None), dict(v=None), dict(k=4104), dict(v=4104), dict(pt=None), dict(lk=None), dict(ws=None), dict(ws=4096 + 512),
              dict(ns=-1), dict(ns=5)]
    if fmt:
        common += [dict(ks=None), dict(vs=None)]
    assert _append(lib, h) == 4 and _decode(lib, h) == 4
    if not fmt:
        assert _append(lib, h, ks=None, vs=None) == 4 and _decode(lib, h, ks=None, vs=None) == 4
    for kw in common + [dict(k_new=None), dict(v_new=None), dict(k_new=4104), dict(v_new=4104), dict(cu=None), dict(total=-1),
                        dict(stride=255), dict(stride=260), dict(stride=128), dict(stride=-256)]:
        assert _append(lib, h, **kw) == 1, kw
    for kw in common + [dict(q=None), dict(q=4104), dict(out=None), dict(out=4104), dict(cu=None), dict(total=-1), dict(w=-1),
                        dict(s=-1), dict(stride=1023), dict(stride=1020), dict(stride=512), dict(stride=-1024)]:
        assert _decode(lib, h, **kw) == 1, kw
    assert _decode(lib, h, total=(1 << 31) - 1) == 3
    if fmt == 0:
        assert _expand(lib, h) == 2      # BF16 pages already
    else:
        assert _expand(lib, h) == 4
        for kw in common + [dict(ko=None), dict(vo=None), dict(ko=4112), dict(vo=4112), dict(opt=None), dict(pages=-1)]:
            assert _expand(lib, h, **kw) == 1, kw
    # nothing to do: fine without a device, and without data
    assert _append(lib, h, total=0, k_new=None, v_new=None) == 0 and _append(lib, h, ns=0) == 0
    assert _decode(lib, h, total=0, q=None, out=None) == 0 and _decode(lib, h, ns=0) == 0
    assert lib.fp2_cache_read_status(h, 4096, None, None) == 4
    cache.close()


def test_binding_refuses_tensors_that_are_not_what_the_address_is_taken_for():
    """Types, shapes, strides and devices are checked where the tensors are still known; nothing is launched."""
    cache = binding.Cache(cache_params(max_seqs=3))
    k, v, ks, vs = cache.new_pages("cpu")
    ws = cache.new_workspace("cpu")
    pt = torch.zeros(3, 32, dtype=torch.int32)
    cu, lk = torch.tensor([0, 1, 2, 3], dtype=torch.int32), torch.tensor([5, 6, 7], dtype=torch.int32)
    q = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    new = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    good = dict(q=q, k_cache=k, v_cache=v, page_table=pt, cu_seqlens_q=cu, seqlens_k=lk, k_scale=ks, v_scale=vs,
                out=torch.zeros_like(q), lse=torch.zeros(8, 3), workspace=ws)
    for name, bad in [("q", q.float()), ("q", q.transpose(0, 1)), ("q", torch.zeros(3, 8, 256, dtype=torch.bfloat16)[:, :, ::2]),
                      ("q", torch.zeros(3, 4, 128, dtype=torch.bfloat16)), ("k_cache", k.to(torch.bfloat16)), ("v_cache", v[:5]),
                      ("page_table", pt.long()), ("page_table", pt[:, :16]), ("cu_seqlens_q", cu[:3]), ("seqlens_k", lk.long()),
                      ("k_scale", ks[0]), ("k_scale", None), ("v_scale", vs.double()), ("out", torch.zeros(2, 8, 128, dtype=torch.bfloat16)),
                      ("out", q.float()), ("lse", torch.zeros(3, 8)), ("workspace", ws[:100])]:
        with pytest.raises(binding.Fp2Error) as e:
            binding.fp2_decode(cache, **{**good, name: bad})
        assert e.value.code == 1, name
    good = dict(k_new=new, v_new=new, page_table=pt, cu_seqlens_new=cu, seqlens_k=lk, k_cache=k, v_cache=v, k_scale=ks, v_scale=vs,
                workspace=ws)
    wide = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    for name, bad in [("k_new", new.half()), ("k_new", wide[:, ::2]), ("v_new", wide[:, :2]), ("v_new", new[:2]),
                      ("cu_seqlens_new", cu.long()), ("k_cache", k.view(-1, 16, 2, 64))]:
        with pytest.raises(binding.Fp2Error) as e:
            binding.fp2_cache_append(cache, **{**good, name: bad})
        assert e.value.code == 1, name
    out = torch.zeros(9, 16, 2, 128, dtype=torch.bfloat16)
    good = dict(k_cache=k, v_cache=v, page_table=pt, seqlens_k=lk, k_scale=ks, v_scale=vs, k_out=out, v_out=out.clone(),
                out_page_table=pt, workspace=ws)
    for name, bad in [("k_out", out.float()), ("v_out", out[:4]), ("out_page_table", pt[:2]), ("k_out", out[:, :8])]:
        with pytest.raises(binding.Fp2Error) as e:
            binding.fp2_cache_expand(cache, **{**good, name: bad})
        assert e.value.code == 1, name
    cache.close()


@pytest.mark.parametrize("window,sinks,code", [(0, 4, 1), (-1, 0, 1), (4, -1, 1), (1, 0, 4), (2 ** 31 - 1, 2 ** 31 - 1, 4)])
def test_window_prefill_refuses(window, sinks, code):
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    prm = dict(num_seqs=1, total_q=300, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=128, tile_rows=128, page_size=16,
               num_pages=64, max_pages_per_seq=32, sink_tokens=256, window_tokens=512, use_correction=1, alpha=0.1,
               softmax_scale=0.0, dtype=1)
    plan = binding.Plan(prm, [0, 300], [400])
    lib, p = binding.load(), C.c_void_p(4096)
    assert lib.fp2_window_prefill(plan.handle, p, p, p, p, p, p, p, p, p, window, sinks, p, None, p, None) == code
    for bad in (dict(q=None), dict(q=4104), dict(out=4112), dict(out=None), dict(ws=512), dict(qs=None), dict(pt=None)):
        a = dict(dict(q=4096, pt=4096, qs=4096, out=4096, ws=4096), **bad)
        assert lib.fp2_window_prefill(plan.handle, a["q"], p, p, a["pt"], p, p, a["qs"], p, p, 16, 0, a["out"], None, a["ws"], None) == 1
    assert lib.fp2_window_prefill(None, p, p, p, p, p, p, p, p, p, 16, 0, p, None, p, None) == 1
    plan.close()


@pytest.mark.parametrize("kw,code", [(dict(num_pages=1 << 27), 3), (dict(num_pages=(1 << 27) - 1), None), (dict(num_pages=1 << 24, page_size=128), 3),
                                     (dict(max_pages_per_seq=1 << 26), None), (dict(num_q_heads=8192, num_kv_heads=1), None),
                                     (dict(num_q_heads=8200, num_kv_heads=1), 3)])
def test_cache_create_at_its_limits(kw, code):
    if code is None:
        binding.Cache(cache_params(**kw)).close()
        return
    with pytest.raises(binding.Fp2Error) as e:
        binding.Cache(cache_params(**kw))
    assert e.value.code == code


@pytest.mark.parametrize("fmt", [0, 1, 2])
def test_an_empty_batch_is_nothing_to_do(fmt):
    """No sequences, as an engine's tensors say it: these have no address."""
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    cache = binding.Cache(cache_params(format=fmt))
    k, v, ks, vs = cache.new_pages(dev)
    ws, pt = cache.new_workspace(dev), torch.zeros(0, 32, dtype=torch.int32, device=dev)
    lk, cu = torch.zeros(0, dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    assert pt.data_ptr() == 0 and lk.data_ptr() == 0
    stream = types.SimpleNamespace(cuda_stream=0)      # (asking torch for one takes a device)
    q, new = torch.zeros(0, 8, 128, dtype=torch.bfloat16, device=dev), torch.zeros(0, 2, 128, dtype=torch.bfloat16, device=dev)
    binding.fp2_cache_append(cache, new, new, pt, cu, lk, k, v, ks, vs, ws, stream=stream)
    binding.fp2_decode(cache, q, k, v, pt, cu, lk, ks, vs, q.clone(), torch.zeros(8, 0, device=dev), ws, stream=stream)
    if fmt:
        out = torch.zeros(0, 16, 2, 128, dtype=torch.bfloat16, device=dev)
        binding.fp2_cache_expand(cache, k, v, pt, lk, ks, vs, out, out.clone(), pt, ws, stream=stream)
    lib = binding.load()
    assert lib.fp2_cache_append(cache.handle, 4096, 4096, 256, None, None, None, 1, 1, 4096, 4096, 4096, 4096, 4096, None) == 1
    assert lib.fp2_decode(cache.handle, 4096, 1024, 4096, 4096, None, None, None, 1, 1, 4096, 4096, 0, 0, 4096, None, 4096, None) == 1
    cache.close()


@pytest.mark.parametrize("fp8", [False, True])
def test_window_prefill_refuses_tensors_that_are_not_what_the_address_is_taken_for(fp8):
    """Queries that are a slice of a fused projection, other types, fewer elements, other row lengths; what has more elements behind
    those of the call goes through (to the lack of a device)."""
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    prm = dict(num_seqs=2, total_q=300, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=128, tile_rows=128, page_size=16,
               num_pages=64, max_pages_per_seq=32, sink_tokens=256, window_tokens=512, use_correction=1, alpha=0.1,
               softmax_scale=0.0, dtype=1 if fp8 else 0)
    plan = binding.Plan(prm, [0, 200, 300], [400, 100])
    kind = torch.uint8 if fp8 else torch.bfloat16
    q, k = torch.zeros(300, 8, 128, dtype=kind), torch.zeros(64, 16, 2, 128, dtype=kind)
    out, lse, pt = torch.zeros(300, 8, 128, dtype=torch.bfloat16), torch.zeros(8, 300), torch.zeros(2, 32, dtype=torch.int32)
    scale = torch.ones(8) if fp8 else None
    good = dict(q=q, k_cache=k, v_cache=k.clone(), page_table=pt, cu_seqlens_q=torch.tensor([0, 200, 300], dtype=torch.int32),
                seqlens_k=torch.tensor([400, 100], dtype=torch.int32), q_scale=scale, k_scale=scale, v_scale=scale, window_tokens=16,
                sink_tokens=0, out=out, lse=lse, workspace=plan.new_workspace("cpu"), stream=types.SimpleNamespace(cuda_stream=0))
    bad = [("q", torch.zeros(300, 12, 128, dtype=kind)[:, :8]), ("q", q.float()), ("q", q[:299]), ("q", torch.zeros(8, 300, 128, dtype=kind).transpose(0, 1)),
           ("k_cache", k[:63]), ("v_cache", k.to(torch.int32)), ("v_cache", torch.zeros(64, 16, 4, 128, dtype=kind)[:, :, ::2]),
           ("page_table", pt.long()), ("page_table", torch.zeros(2, 40, dtype=torch.int32)), ("page_table", torch.zeros(2, 40, dtype=torch.int32)[:, :32]),
           ("out", torch.zeros(300, 16, 128, dtype=torch.bfloat16)[:, :8]), ("out", out.float()), ("out", out[1:]), ("lse", lse.T), ("lse", torch.zeros(8, 400)),
           ("lse", lse.double()), ("workspace", good["workspace"][:64])]
    bad += [(name, None) for name in ("q", "k_cache", "v_cache", "page_table", "out", "workspace")]
    if fp8:
        bad += [("q_scale", None), ("q_scale", torch.ones(7)), ("k_scale", torch.ones(2).double()), ("v_scale", torch.ones(4)[::2])]
    for name, value in bad:
        with pytest.raises(binding.Fp2Error) as e:
            binding.fp2_window_prefill(plan, **{**good, name: value})
        assert e.value.code == 1, (name, value.shape if value is not None else None)
    more = dict(page_table=torch.zeros(5, 32, dtype=torch.int32), q=torch.zeros(400, 8, 128, dtype=kind), out=torch.zeros(400, 8, 128, dtype=torch.bfloat16), k_cache=torch.zeros(70, 16, 2, 128, dtype=kind))
    for kw in ({}, more, dict(lse=None), dict(k_cache=k.view(-1, 2, 128))):
        with pytest.raises(binding.Fp2Error) as e:
            binding.fp2_window_prefill(plan, **{**good, **kw})
        assert e.value.code == 4
    plan.close()


def test_window_prefill_without_new_tokens_is_nothing_to_do():
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    prm = dict(num_seqs=2, total_q=0, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=128, tile_rows=128, page_size=16,
               num_pages=64, max_pages_per_seq=32, sink_tokens=256, window_tokens=512, use_correction=1, alpha=0.1,
               softmax_scale=0.0, dtype=0)
    plan = binding.Plan(prm, [0, 0, 0], [400, 0])
    q, k = torch.zeros(0, 8, 128, dtype=torch.bfloat16, device=dev), torch.zeros(64, 16, 2, 128, dtype=torch.bfloat16, device=dev)
    ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device=dev)
    binding.fp2_window_prefill(plan, q, k, k.clone(), ints(2, 32), ints(3), ints(2), None, None, None, 16, 0, q.clone(),
                               torch.zeros(8, 0, device=dev), plan.new_workspace(dev), stream=types.SimpleNamespace(cuda_stream=0))
    assert plan.last_launch_count() == 0
    assert binding.load().fp2_window_prefill(plan.handle, *[None] * 9, 0, 0, None, None, None, None) == 1      # (a window all the same)
    plan.close()
