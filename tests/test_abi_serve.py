"""The entry points of the 4-bit cache, eviction and sampling without a GPU: their host validation under
AddressSanitizer and UndefinedBehaviorSanitizer (every rejection, and past validation into stubbed launches), the
refusals of the built library, and those of the Python functions."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2606_24957_amd as D

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_24957_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FAKE = 0x10000  # a non-null, 256-byte aligned address that validation never dereferences


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_validation_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "abi_rejections_serve")
    # host code only is instrumented (each -fsanitize= behind -Xarch_host)
    cmd = [HIPCC, "--offload-arch=gfx950", "-x", "hip", "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "api_kv4.hip"),
           os.path.join(CSRC, "api_sample.hip"),
           os.path.join(ROOT, "tests", "sanitize", "abi_rejections_serve.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    out = run.stdout + run.stderr
    assert run.returncode == 0, out[-4000:]
    assert "ok: 0 failed expectations" in out
    for report in ("ERROR: AddressSanitizer", "runtime error:", "ERROR: LeakSanitizer", "UndefinedBehaviorSanitizer"):
        assert report not in out, out[-4000:]


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(D.LIB_PATH):
        pytest.skip("libdustin.so not built")
    return D.lib()


def _batch(B=2, max_len=100, nq=4, k_max=40):
    bt = D.DustinBatch()
    bt.batch, bt.max_len, bt.nq_max, bt.k_max, bt.seq_lens = B, max_len, nq, k_max, FAKE
    return bt


def _kv4(n=200, H=2, d=128):
    kv = D.DustinKV4()
    kv.data = kv.scales = FAKE
    kv.num_kv_heads, kv.head_dim, kv.capacity = H, d, n
    kv.stride_h, kv.stride_n, kv.stride_b = d // 2, H * d // 2, n * H * d // 2
    kv.scale_stride_h, kv.scale_stride_n, kv.scale_stride_b = d // 32, H * d // 32, n * H * d // 32
    return kv


def test_the_built_library_refuses(L):
    r = ctypes.byref
    rows = (FAKE, 1024, 256, 128, FAKE, 1024, 256, 128)
    for fn in (L.dustin_kv4_append, L.dustin_kv4_read):
        assert fn(*rows, r(_kv4()), r(_kv4(H=4)), r(_batch()), None) == D.ERR_INVALID_ARG
        assert fn(*rows, r(_kv4(n=103)), r(_kv4(n=103)), r(_batch()), None) == D.ERR_INVALID_ARG
        assert fn(*rows, r(_kv4(d=96)), r(_kv4(d=96)), r(_batch()), None) == D.ERR_UNSUPPORTED
    attn = lambda kv, bt, Hq=8, ws=FAKE, n=1 << 40: L.dustin_dense_verify_attn_kv4(
        FAKE, 4096, 1024, 128, Hq, r(kv), r(kv), r(bt), 0.1, FAKE, 4096, 1024, 128, ws, n, None)
    assert attn(_kv4(), _batch(), Hq=7) == D.ERR_INVALID_ARG
    assert attn(_kv4(d=64), _batch()) == D.ERR_UNSUPPORTED
    assert attn(_kv4(), _batch(nq=33)) == D.ERR_UNSUPPORTED
    assert attn(_kv4(), _batch(), ws=None) == D.ERR_WORKSPACE
    assert attn(_kv4(), _batch(), n=64) == D.ERR_WORKSPACE
    s = D.DustinSampling(float("nan"), 0, 1.0, 0.0, None, None, None, None)
    draw = lambda V=100, ws=FAKE, n=1 << 40: L.dustin_sample(FAKE, 0, V, 1, V, r(s), FAKE, FAKE, None, 0, ws, n, None)
    assert draw() == D.ERR_INVALID_ARG
    s.temperature = 1.0
    assert draw(V=(1 << 18) + 1) == D.ERR_UNSUPPORTED
    assert draw(ws=None) == D.ERR_WORKSPACE and draw(n=64) == D.ERR_WORKSPACE


def test_views_of_4_bit_caches():
    k, v = D.kv4_empty(3, 20, 2, 128, "cpu")
    assert k.data.shape == v.data.shape == (3, 20, 2, 64) and k.scales.shape == (3, 20, 2, 4)
    a, b = D.kv4_view(k), D.kv4_view(v)
    assert b.data - a.data == 64 and a.stride_h == 128 and a.stride_n == 256 and a.capacity == 20
    assert b.scales - a.scales == 4 and a.scale_stride_h == 8
    table = torch.zeros(5, 7, dtype=torch.int32)
    p = D.kv4_view(k, table)
    assert (p.page_size, p.max_pages, p.num_pages, p.stride_page) == (20, 7, 3, 20 * 256)
    with pytest.raises(ValueError, match="page_table"):
        D.kv4_view(k, table.long())
    with pytest.raises(ValueError, match="uint8"):
        D.kv4_view(D.KV4(k.data.float(), k.scales))
    with pytest.raises(ValueError, match="contiguous rows"):
        D.kv4_view(D.KV4(k.data.transpose(2, 3), k.scales))
    with pytest.raises(ValueError, match="do not belong"):
        D.kv4_view(D.KV4(k.data[:2], k.scales))


def test_host_tensors_are_refused():
    k, v = D.kv4_empty(1, 20, 2, 128, "cpu")
    rows = torch.zeros(1, 2, 2, 128, dtype=torch.bfloat16)
    idx, cnt = torch.zeros(1, 1, 4, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32)
    u = torch.zeros(1)
    if torch.cuda.is_available():
        pytest.skip("the device is there: the refusals below are those of a host without one as well")
    for call in (lambda: D.kv4_append(rows, rows, k, v, [0]), lambda: D.dense_verify_attn_kv4(rows, k, v, [0]),
                 lambda: D.sparse_verify_attn_kv4(rows, k, v, idx, cnt, [0]), lambda: D.kv_evict(k, v, idx, cnt),
                 lambda: D.sample(torch.zeros(1, 9), u),
                 lambda: D.verify_tokens(torch.zeros(1, 2, 9), idx[:, 0, :1], u.view(1, 1), u)):
        with pytest.raises(ValueError, match="GPU only"):
            call()
    with pytest.raises(ValueError, match="both outputs"):
        D.kv4_read(k, v, [0], k_out=rows)
    with pytest.raises(ValueError, match="needs nq_max"):
        D.kv4_read(k, v, [0])
    b = rows
    with pytest.raises(ValueError, match="one cache"):
        D.kv_evict(k, k, idx, cnt)
    with pytest.raises(ValueError, match="or KV4"):
        D.kv_evict(k, b, idx, cnt)
    with pytest.raises(ValueError, match="outputs for each"):
        D.kv_evict(k, v, idx, cnt, k_out=k)
    with pytest.raises(ValueError, match="outputs for each"):
        D.kv_evict(k, None, idx, cnt, v_out=v)
    with pytest.raises(ValueError, match="out_page_table"):
        D.kv_evict(k, v, idx, cnt, out_page_table=idx[0])
