"""Refusals of the context-cache operators, through the C ABI and the binding,
and their host layer under sanitizers: no GPU is used, and no placeholder
pointer is ever read (every call that reaches the library fails its checks)."""

import ctypes
import os
import shutil
import subprocess
import types

import pytest
import torch

import paper_2609_00355_amd as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "host_sanitize")
ROCM_INCLUDE = "/opt/rocm/include"
FAKE = 0x10000
BAD, UNSUP, WS = G.GLANCE_ERR_INVALID_ARG, G.GLANCE_ERR_UNSUPPORTED, G.GLANCE_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(G.LIB_PATH):
        from paper_2609_00355_amd import build
        build.build()
    return G.lib()


def _cache(at=1, **kw):
    base = dict(batch=1, n_kv_heads=4, head_dim=128, capacity=512, format=G.GLANCE_CACHE_DENSE, dtype=G.GLANCE_BF16,
                k=at << 40, v=(at + 1) << 40, k_scale=None, v_scale=None, ctx_lens=FAKE, weights=(at + 2) << 40)
    base.update(kw)
    return G.CacheStruct(**base)


def _kv4(at=1, **kw):
    return _cache(at, **{**dict(format=G.GLANCE_CACHE_KV4, k_scale=(at + 3) << 40, v_scale=(at + 4) << 40), **kw})


def _shape(**kw):
    base = dict(batch=1, n_new=16, n_q_heads=28, n_kv_heads=4, head_dim=128, ctx_capacity=512, dtype=G.GLANCE_BF16)
    base.update(kw)
    return G.attn_shape(**base)


def _attn(lib, cache, shape=None, n_sinks=0, window=64, q=FAKE, k_new=FAKE, v_new=FAKE, parents=FAKE, out=FAKE, ws=FAKE, ws_bytes=0):
    s = shape or _shape()
    return lib.glance_cache_tree_verify_attn(ctypes.byref(s), ctypes.byref(cache) if cache else None, n_sinks, window, q, k_new, v_new,
                                             parents, out, None, ws, ws_bytes, None)


@pytest.mark.parametrize("cache,kw,code,word", [
    (None, {}, BAD, "cache is NULL"),
    (_cache(batch=0), {}, BAD, "batch"),
    (_cache(batch=2), {}, BAD, "the shape's"),
    (_cache(batch=40000), {}, UNSUP, "batch"),
    (_cache(n_kv_heads=0), {}, BAD, "n_kv_heads"),
    (_cache(head_dim=96), {}, UNSUP, "head_dim"),
    (_cache(head_dim=64), {}, BAD, "the shape's"),
    (_cache(capacity=-1), {}, BAD, "capacity"),
    (_cache(capacity=2 ** 25 + 1), {}, UNSUP, "capacity"),
    (_cache(capacity=500), {}, BAD, "the shape's"),
    (_cache(format=2), {}, UNSUP, "format"),
    (_cache(dtype=7), {}, UNSUP, "dtype"),
    (_cache(dtype=G.GLANCE_F32), {}, BAD, "dtype"),
    (_cache(k=None), {}, BAD, "cache: k is NULL"),
    (_cache(v=8), {}, BAD, "cache: v is not 16-byte aligned"),
    (_cache(ctx_lens=None), {}, BAD, "ctx_lens"),
    (_kv4(k_scale=None), {}, BAD, "k_scale"),
    (_kv4(v_scale=0x10004), {}, BAD, "v_scale"),
    (_kv4(), dict(n_sinks=-1), BAD, "n_sinks"),
    (_kv4(), dict(window=-1), BAD, "window"),
    (_kv4(), dict(q=None), BAD, "q"),
    (_kv4(), dict(parents=None), BAD, "parents"),
    (_kv4(), dict(out=0x10008), BAD, "out"),
    (_kv4(), dict(ws=None), WS, "workspace"),
    (_kv4(), dict(ws_bytes=255), WS, "too small"),
    (_kv4(), dict(shape=_shape(n_new=65)), UNSUP, "n_new"),
])
def test_attention_refusals(lib, cache, kw, code, word):
    assert _attn(lib, cache, **kw) == code, G.glance_last_error()
    assert word in G.glance_last_error()


def test_workspace_size(lib):
    assert G.glance_cache_attn_workspace_size(_shape(), 0, 0) > 0
    assert G.glance_cache_attn_workspace_size(_shape(), -1, 0) == 0
    assert G.glance_cache_attn_workspace_size(_shape(), 0, -1) == 0
    assert G.glance_cache_attn_workspace_size(_shape(n_new=0), 0, 0) == 0


@pytest.mark.parametrize("src,dst,code,word", [
    (None, _kv4(), BAD, "src is NULL"),
    (_cache(), None, BAD, "dst is NULL"),
    (_cache(), _cache(16), BAD, "4 bits"),
    (_kv4(), _kv4(16), BAD, "4 bits"),
    (_cache(), _kv4(16, n_kv_heads=2), BAD, "same batch"),
    (_cache(), _kv4(16, head_dim=64), BAD, "same batch"),
    (_cache(), _kv4(16, k=(2 << 40) + 64), BAD, "overlap"),
    (_cache(), _kv4(16, k_scale=(1 << 40) + 4 * 512 * 256 - 16), BAD, "overlap"),
])
def test_convert_refusals(lib, src, dst, code, word):
    assert lib.glance_cache_convert(ctypes.byref(src) if src else None, ctypes.byref(dst) if dst else None, None) == code
    assert word in G.glance_last_error()


@pytest.mark.parametrize("cache,kw,code,word", [
    (_kv4(), dict(n=0), UNSUP, "n_nodes"),
    (_kv4(), dict(n=65), UNSUP, "n_nodes"),
    (_kv4(), dict(dtype=3), UNSUP, "dtype"),
    (_kv4(capacity=0), {}, BAD, "capacity"),
    (_kv4(), dict(stride=0), BAD, "path_stride"),
    (_kv4(), dict(k_new=None), BAD, "k_new"),
    (_kv4(), dict(k_new=0x10008), BAD, "aligned"),
    (_kv4(), dict(path=None), BAD, "accept_path"),
    (_cache(), dict(dtype=G.GLANCE_F32), BAD, "dtype"),
    (_cache(), dict(n=65), UNSUP, "n_nodes"),
])
def test_commit_refusals(lib, cache, kw, code, word):
    a = dict(n=8, dtype=G.GLANCE_BF16, k_new=FAKE, v_new=FAKE, alen=FAKE, path=FAKE, stride=8)
    a.update(kw)
    assert lib.glance_cache_commit_path(ctypes.byref(cache), a["n"], a["dtype"], a["k_new"], a["v_new"], a["alen"], a["path"],
                                        a["stride"], None) == code
    assert word in G.glance_last_error()


@pytest.mark.parametrize("cache,kw,code,word", [
    (_kv4(), dict(decay=-0.1), BAD, "decay"),
    (_kv4(), dict(decay=1.1), BAD, "decay"),
    (_kv4(), dict(decay=float("nan")), BAD, "decay"),
    (_kv4(weights=None), dict(decay=0.5), BAD, "weights"),
    (_kv4(), dict(lse=None), BAD, "lse"),
    (_kv4(), dict(out=None), BAD, "weights_out"),
    (_kv4(), dict(out=(3 << 40) + 4), BAD, "apart"),
    (_kv4(), dict(k_new=FAKE), BAD, "path"),
    (_kv4(), dict(path=FAKE, alen=FAKE), BAD, "path"),
    (_kv4(), dict(path=FAKE, k_new=FAKE), BAD, "path"),
    (_kv4(), dict(path=FAKE, alen=FAKE, k_new=FAKE, stride=0), BAD, "path_stride"),
    (_kv4(), dict(window=-5), BAD, "window"),
    (_kv4(batch=3), {}, BAD, "the shape's"),
])
def test_weigh_refusals(lib, cache, kw, code, word):
    a = dict(n_sinks=0, window=0, q=FAKE, lse=FAKE, k_new=None, alen=None, path=None, stride=8, decay=1.0, out=5 << 44)
    a.update(kw)
    s = _shape()
    assert lib.glance_cache_weigh(ctypes.byref(s), ctypes.byref(cache), a["n_sinks"], a["window"], a["q"], a["lse"], a["k_new"],
                                  a["alen"], a["path"], a["stride"], a["decay"], a["out"], None) == code, G.glance_last_error()
    assert word in G.glance_last_error()
    empty, s0 = _cache(capacity=0), _shape(ctx_capacity=0)
    assert lib.glance_cache_weigh(ctypes.byref(s0), ctypes.byref(empty), 0, 0, FAKE, FAKE, None, None, None, 0, 0.0, FAKE, None) == BAD


@pytest.mark.parametrize("src,dst,kw,code,word", [
    (_cache(), _kv4(16), {}, BAD, "same format"),
    (_cache(), _cache(16, dtype=G.GLANCE_F32), {}, BAD, "same format"),
    (_cache(weights=None), _cache(16), {}, BAD, "src: weights"),
    (_cache(), _cache(16, weights=None), {}, BAD, "dst: weights"),
    (_cache(), _cache(16), dict(budget=0), BAD, "budget"),
    (_cache(), _cache(16), dict(budget=513), BAD, "capacity"),
    (_cache(), _cache(16), dict(n_sinks=-1), BAD, "n_sinks"),
    (_cache(), _cache(16), dict(n_sinks=60, n_recent=41), BAD, "budget"),
    (_cache(), _cache(16), dict(n_sinks=2 ** 31 - 1, n_recent=2 ** 31 - 1), BAD, "budget"),
    (_cache(), _cache(16), dict(kept=None), BAD, "kept"),
    (_cache(), _cache(1), {}, BAD, "overlap"),
    (_cache(), _cache(16, weights=1 << 40), {}, BAD, "overlap"),
    (_cache(capacity=0), _cache(16), {}, BAD, "capacity"),
    (_cache(batch=300, n_kv_heads=300, capacity=1), _cache(16, batch=300, n_kv_heads=300, capacity=200), {}, UNSUP, "65535"),
])
def test_evict_refusals(lib, src, dst, kw, code, word):
    a = dict(budget=100, n_sinks=0, n_recent=0, kept=FAKE)
    a.update(kw)
    assert lib.glance_cache_evict(ctypes.byref(src), ctypes.byref(dst), a["budget"], a["n_sinks"], a["n_recent"], a["kept"], None) == code
    assert word in G.glance_last_error()


def test_lengths_that_overlap_in_part_are_refused(lib):
    src, conv, ev = _cache(batch=4), _kv4(16, batch=4, ctx_lens=FAKE + 8), _cache(16, batch=4, ctx_lens=FAKE - 12)
    assert lib.glance_cache_convert(ctypes.byref(src), ctypes.byref(conv), None) == BAD
    assert "ctx_lens" in G.glance_last_error()
    assert lib.glance_cache_evict(ctypes.byref(src), ctypes.byref(ev), 100, 0, 0, FAKE, None) == BAD
    assert "ctx_lens" in G.glance_last_error()


def test_binding_refusals():
    """What the binding turns away before it calls the library, on host tensors."""
    cache = G.new_cache(1, 2, 8, 64, fmt="kv4", weights=True, device="cpu")
    assert cache.kv4 and (cache.batch, cache.n_kv_heads, cache.capacity, cache.head_dim) == (1, 2, 8, 64)
    q = torch.zeros(1, 4, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        G.glance_cache_block_draft_attn(q, cache, q, q)
    with pytest.raises(ValueError, match="GPU"):
        G.glance_cache_convert(cache, cache)
    with pytest.raises(ValueError, match="fmt"):
        G.new_cache(1, 2, 8, 64, fmt="int4", device="cpu")
    with pytest.raises(ValueError, match="32"):
        G.new_cache(1, 2, 8, 80, fmt="kv4", device="cpu")
    assert G.new_cache(1, 2, 8, 64, device="cpu").k.dtype == torch.bfloat16


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32, 2 ** 32 + 8, -2 ** 31 - 1])
def test_numbers_past_32_bits_are_refused(lib, big):
    """The library's are 32 bits: cut to them, 2^32 would be no window and 2^32 + 8 one of 8."""
    cache = G.new_cache(1, 2, 8, 64, weights=True, device="cpu")
    q, lse = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 1, 2)
    for kw in (dict(n_sinks=big), dict(window=big)):
        with pytest.raises(ValueError, match=f"{next(iter(kw))} must fit 32 bits"):
            G.glance_cache_attn_workspace_size(_shape(), **kw)
        for call in (lambda: G.glance_cache_block_draft_attn(q, cache, q, q, **kw),
                     lambda: G.prepare_cache_tree_verify_attn(q, cache, q, q, None, **kw),
                     lambda: G.glance_cache_weigh(q, cache, lse, **kw)):
            with pytest.raises(ValueError, match="must fit 32 bits"):
                call()
    for kw in (dict(budget=big), dict(budget=4, n_sinks=big), dict(budget=4, n_recent=big)):
        with pytest.raises(ValueError, match="must fit 32 bits"):
            G.glance_cache_evict(cache, cache, **kw)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The calls run on the current device: a tensor elsewhere would be read by the wrong GPU."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    here, there = (types.SimpleNamespace(device=torch.device("cuda", i)) for i in (0, 1))
    G._same_device(here, None, here)
    with pytest.raises(ValueError, match="cuda:1"):
        G._same_device(here, there)


def test_host_layer_under_asan_and_ubsan(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir(os.path.join(ROCM_INCLUDE, "hip")):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "cache_driver")
    csrc = os.path.join(ROOT, "paper_2609_00355_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-g", "-O1", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INCLUDE, "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", HERE,
           os.path.join(csrc, "glance_api.cpp"), os.path.join(csrc, "glance_cache_api.cpp"), os.path.join(HERE, "stubs.cpp"),
           os.path.join(HERE, "cache_stubs.cpp"), os.path.join(HERE, "cache_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "checks passed" in r.stdout
