"""CPU-side checks of 4-bit caches, attention weights, eviction and 4-bit products: bad host-visible arguments are refused with the documented status
before anything is launched (the addresses are fake and never dereferenced), calls without work are no-ops, and the host code is clean under the address and
undefined-behaviour sanitizers."""
from __future__ import annotations

import os
import subprocess

import pytest

import paper_2603_02631_amd as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FAKE = 0x10000


class OnGpu:
    """A tensor of the CPU that says it is on the GPU: the binding looks at it, the library refuses the call before anything is read."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)

    def data_ptr(self):
        return FAKE


def cache(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, cache_type=sp.SP_CACHE_MX4, n_pages=4, page_tokens=64, page_stride=2 * 64 * 64, stride_head=64 * 64,
                stride_token=64)
    base.update(kw)
    return sp.CacheDesc(*[base[f[0]] for f in sp.CacheDesc._fields_])


def refused(status, fn, *args, **kw):
    with pytest.raises(sp.SpError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value
    assert e.value.message
    return e.value.message


def append(d=None, **kw):
    a = dict(k=FAKE, v=FAKE, offsets_host=[0, 3], offsets_dev=FAKE, start=FAKE, block_table=FAKE, k_pool=FAKE, v_pool=FAKE, k_scale=FAKE, v_scale=FAKE, q=FAKE,
             q_out=FAKE, cos=FAKE, sin=FAKE, n_pos=100, rot_dim=64, rot_style=0, table_stride=4, stream=0)
    a.update(kw)
    sp.sp_cache_append(d or cache(), **a)


def attend(d=None, **kw):
    a = dict(q=FAKE, offsets_host=[0, 3, 4], offsets_dev=FAKE, lens=FAKE, max_len=200, block_table=FAKE, k_pool=FAKE, v_pool=FAKE, k_scale=FAKE, v_scale=FAKE,
             scale=0.125, out=FAKE, lse=FAKE, ws=FAKE, causal=1, window=0, table_stride=4, ws_bytes=1 << 40, stream=0)
    a.update(kw)
    sp.sp_attend(d or cache(), **a)


def weights(d=None, **kw):
    a = dict(q=FAKE, offsets_host=[0, 3, 4], offsets_dev=FAKE, lens=FAKE, max_len=200, block_table=FAKE, k_pool=FAKE, k_scale=FAKE, scale=0.125, lse=FAKE, old=FAKE,
             weights=FAKE, causal=1, window=0, table_stride=4, weights_stride=200, stream=0)
    a.update(kw)
    sp.sp_attend_weights(d or cache(), **a)


def evict(d=None, **kw):
    a = dict(lens=FAKE, max_len=200, budget=FAKE, max_budget=100, sinks=4, recent=8, weights=FAKE, block_table=FAKE, dst_table=FAKE, k_pool=FAKE, v_pool=FAKE,
             k_scale=FAKE, v_scale=FAKE, new_lens=FAKE + 64, kept=FAKE, new_weights=FAKE + 4096, B=2, weights_stride=200, table_stride=4, dst_stride=2, stream=0)
    a.update(kw)
    sp.sp_cache_evict(d or cache(), **a)


def quantise(**kw):
    a = dict(x=FAKE, rows=3, K=96, codes=FAKE, scales=FAKE, dtype=sp.SP_LOGITS_BF16, row_stride=96, stream=0)
    a.update(kw)
    sp.sp_mx4_quantise(**a)


def matmul(**kw):
    a = dict(a_codes=FAKE, a_scales=FAKE, M=3, w_codes=FAKE, w_scales=FAKE, N=5, K=96, out=FAKE, dtype=sp.SP_LOGITS_BF16, out_stride=5, stream=0)
    a.update(kw)
    sp.sp_mx4_matmul(**a)


@pytest.mark.parametrize("kw,status", [
    (dict(stride_token=80), 1), (dict(stride_token=72), 1), (dict(stride_head=64 * 64 + 16), 1), (dict(page_stride=2 * 64 * 64 + 8), 1), (dict(head_dim=96), 2),
    (dict(cache_type=4), 1), (dict(cache_type=-1), 1), (dict(page_tokens=48), 1), (dict(n_kv_heads=3), 1)])
def test_descriptions_of_4_bit_caches(kw, status):
    d = cache(**kw)
    refused(status, sp.sp_attend_workspace, d, [0, 1], 1, 64)
    for fn in (append, attend, weights, evict):
        refused(status, fn, d)


def test_strides_of_4_bit_caches_are_multiples_of_32():
    assert sp.sp_attend_workspace(cache(stride_token=96, stride_head=96 * 64, page_stride=2 * 96 * 64), [0, 1], 1, 64) >= 0


@pytest.mark.parametrize("fn", [append, attend, evict])
@pytest.mark.parametrize("kw", [dict(k_scale=None), dict(v_scale=None), dict(k_scale=FAKE + 4), dict(v_scale=FAKE + 8), dict(k_pool=FAKE + 8), dict(v_pool=None)])
def test_pools_and_scales_of_4_bit_caches(fn, kw):
    refused(1, fn, **kw)


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(lse=None), dict(weights=None), dict(offsets_dev=None), dict(lens=None), dict(block_table=None), dict(k_pool=None), dict(k_scale=None),
    dict(q=FAKE + 8), dict(k_pool=FAKE + 8), dict(k_scale=FAKE + 2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
    dict(scale=2.4e38), dict(causal=2), dict(causal=-1), dict(window=-1), dict(causal=0, window=5), dict(max_len=257, weights_stride=257), dict(max_len=-1),
    dict(max_len=(1 << 30) + 1, table_stride=1 << 30, weights_stride=1 << 31), dict(table_stride=0), dict(table_stride=(1 << 31) + 1), dict(offsets_host=[0, 4, 3]),
    dict(offsets_host=[2, 3]), dict(weights_stride=199), dict(weights_stride=-1), dict(weights_stride=(1 << 40) + 1), dict(offsets_host=[0] * 4098)])
def test_weights_refuse(kw):
    refused(1, weights, **kw)


def test_weights_refuse_more_than_a_launch_holds():
    refused(2, weights, cache(n_q_heads=4096, n_kv_heads=4096), offsets_host=[0] * 17)
    refused(2, weights, offsets_host=[0, (1 << 26) + 1])


def test_weights_of_nothing_are_a_no_op():
    weights(offsets_host=[0], q=None, weights=None, lens=None)
    weights(max_len=0, q=None, weights=None, lse=None)


@pytest.mark.parametrize("kw", [
    dict(lens=None), dict(budget=None), dict(weights=None), dict(block_table=None), dict(dst_table=None), dict(new_lens=None), dict(kept=None), dict(k_pool=None),
    dict(B=-1), dict(B=4097), dict(max_len=-1), dict(max_len=257, weights_stride=257), dict(max_len=(1 << 30) + 1, table_stride=1 << 30, weights_stride=1 << 31),
    dict(max_budget=-1), dict(max_budget=(1 << 30) + 1), dict(sinks=-1), dict(recent=-1), dict(table_stride=0), dict(dst_stride=0), dict(dst_stride=(1 << 31) + 1),
    dict(weights_stride=199), dict(weights_stride=(1 << 40) + 1), dict(new_weights=FAKE), dict(new_lens=FAKE)])
def test_evict_refuses(kw):
    refused(1, evict, **kw)


def test_evict_refuses_what_would_be_overwritten_while_it_is_read():
    assert "lens_dev" in refused(1, evict, new_lens=FAKE, budget=FAKE + 256)
    assert "budget_dev" in refused(1, evict, new_lens=FAKE, lens=FAKE + 256)
    assert "weights_dev" in refused(1, evict, new_weights=FAKE)


def test_evict_refuses_more_than_a_launch_holds():
    refused(2, evict, cache(n_q_heads=4096, n_kv_heads=4096), B=17)
    for n in (1 << 29, (1 << 29) - 31):
        refused(2, evict, max_len=n, max_budget=n, weights_stride=n, table_stride=1 << 24)


def test_evict_of_nothing_is_a_no_op():
    evict(B=0, lens=None, weights=None, kept=None, new_lens=None)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(codes=None), dict(scales=None), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(K=0), dict(K=-32), dict(K=48),
    dict(K=1 << 31, row_stride=1 << 31), dict(row_stride=64), dict(row_stride=100), dict(row_stride=(1 << 40) + 8), dict(x=FAKE + 8), dict(codes=FAKE + 8),
    dict(scales=FAKE + 2)])
def test_quantise_refuses(kw):
    refused(1, quantise, **kw)


@pytest.mark.parametrize("kw", [
    dict(a_codes=None), dict(a_scales=None), dict(w_codes=None), dict(w_scales=None), dict(out=None), dict(dtype=2), dict(dtype=-1), dict(M=-1), dict(N=-1),
    dict(M=1 << 31), dict(N=1 << 31, out_stride=1 << 31), dict(K=0), dict(K=-32), dict(K=40), dict(K=1 << 31), dict(out_stride=4), dict(out_stride=(1 << 40) + 1),
    dict(a_codes=FAKE + 8), dict(w_codes=FAKE + 4), dict(a_scales=FAKE + 2), dict(w_scales=FAKE + 1), dict(out=FAKE + 1),
    dict(out=FAKE + 2, dtype=sp.SP_LOGITS_F32)])
def test_matmul_refuses(kw):
    refused(1, matmul, **kw)


def test_products_refuse_more_than_a_launch_holds():
    refused(2, quantise, rows=1 << 30, K=64, row_stride=64)
    refused(2, matmul, M=1 << 17, N=1 << 17, out_stride=1 << 17)


def test_products_of_nothing_are_no_ops():
    quantise(rows=0, x=None, codes=None)
    matmul(M=0, a_codes=None, out=None)
    matmul(N=0, out_stride=0, w_codes=None)
    refused(1, quantise, rows=0, K=40)                          # the sizes are looked at all the same
    refused(1, matmul, M=0, K=40)


def test_an_address_needs_what_a_tensor_would_say():
    refused(1, quantise, dtype=None)
    refused(1, matmul, dtype=None)
    refused(1, evict, B=None)


def stops():
    return {append: dict(rot_dim=8, offsets_host=[0, 2, 3]), attend: dict(causal=2), weights: dict(causal=2), evict: dict(sinks=-1), quantise: dict(K=40, row_stride=None),
            matmul: dict(K=40, out_stride=None)}


INDICES = [(weights, "lens", 2, 32), (weights, "block_table", 8, 32), (weights, "offsets_dev", 3, 64), (evict, "lens", 2, 32), (evict, "budget", 2, 32),
           (evict, "block_table", 8, 32), (evict, "dst_table", 4, 32), (evict, "new_lens", 2, 32), (evict, "kept", 400, 32)]


@pytest.mark.parametrize("fn,name,n,bits", INDICES)
def test_indices_of_another_width_are_refused(fn, name, n, bits):
    import torch
    own, other = (torch.int32, torch.int64) if bits == 32 else (torch.int64, torch.int32)
    assert name not in refused(1, fn, **{**stops()[fn], name: OnGpu(torch.zeros(n, dtype=own))})
    for dtype in (other, torch.float32, torch.float64, torch.int16):
        assert name in refused(1, fn, **{**stops()[fn], name: OnGpu(torch.zeros(4 * n, dtype=dtype))})


NUMBERS = [(weights, "q", (4, 8, 64), "bfloat16"), (weights, "lse", (4, 8), "float32"), (weights, "weights", (2, 2, 200), "float32"), (weights, "old", (2, 2, 200), "float32"),
           (weights, "k_pool", (4, 2, 64, 32), "uint8"), (weights, "k_scale", (4, 2, 64, 2), "uint8"), (attend, "k_pool", (4, 2, 64, 32), "uint8"),
           (attend, "v_scale", (4, 2, 64, 2), "uint8"), (append, "k_pool", (4, 2, 64, 32), "uint8"), (append, "v_scale", (4, 2, 64, 2), "uint8"),
           (evict, "weights", (2, 2, 200), "float32"), (evict, "new_weights", (2, 2, 100), "float32"), (evict, "v_pool", (4, 2, 64, 32), "uint8"),
           (evict, "k_scale", (4, 2, 64, 2), "uint8"), (quantise, "codes", (3, 48), "uint8"), (quantise, "scales", (3, 3), "uint8"), (matmul, "a_codes", (3, 48), "uint8"),
           (matmul, "a_scales", (3, 3), "uint8"), (matmul, "w_codes", (5, 48), "uint8"), (matmul, "w_scales", (5, 3), "uint8")]


@pytest.mark.parametrize("fn,name,shape,own", NUMBERS)
def test_numbers_of_another_type_are_refused(fn, name, shape, own):
    import torch
    for dtype in (own, {"bfloat16": "int16", "float32": "int32", "uint8": "int8"}[own]):
        assert not refused(1, fn, **{**stops()[fn], name: OnGpu(torch.zeros(shape, dtype=getattr(torch, dtype)))}).startswith(name + " ")
    for dtype in {"bfloat16": ("float16", "float32"), "float32": ("float64", "bfloat16"), "uint8": ("float32", "float8_e4m3fn", "int32")}[own]:
        big = (*shape[:-1], 4 * shape[-1]) if own == "uint8" else shape
        message = refused(1, fn, **{**stops()[fn], name: OnGpu(torch.zeros(big, dtype=getattr(torch, dtype)))})
        assert message.startswith(name + " "), message


@pytest.mark.parametrize("fn,name,shape", [(weights, "q", (3, 8, 64)), (weights, "lse", (3, 8)), (weights, "k_pool", (3, 2, 64, 32)), (weights, "k_scale", (4, 2, 64, 1)),
                                           (evict, "kept", (2, 2, 99)), (evict, "new_weights", (2, 2, 99)), (matmul, "w_codes", (4, 48)), (matmul, "a_scales", (2, 3)),
                                           (quantise, "codes", (2, 48)), (quantise, "scales", (3, 2))])
def test_tensors_that_are_too_short_are_refused(fn, name, shape):
    import torch
    dtype = dict(q=torch.bfloat16, lse=torch.float32, kept=torch.int32, new_weights=torch.float32).get(name, torch.uint8)
    stop = {quantise: {}, matmul: {}}.get(fn, stops()[fn])
    message = refused(1, fn, **{**stop, name: OnGpu(torch.zeros(shape, dtype=dtype))})
    assert message.startswith(name + " "), message


def test_weights_and_old_of_different_shape_are_refused():
    import torch
    a, b = OnGpu(torch.zeros(2, 2, 200)), OnGpu(torch.zeros(2, 2, 208))
    assert "shape" in refused(1, weights, weights=a, old=b, weights_stride=None)


@pytest.mark.parametrize("fn,name", [(quantise, "x"), (matmul, "out")])
def test_numbers_of_a_product_of_another_type_are_refused(fn, name):
    import torch
    for dtype in (torch.float16, torch.float64, torch.int64):
        for given in (None, sp.SP_LOGITS_BF16, sp.SP_LOGITS_F32):
            t = torch.zeros(3, 96 if name == "x" else 5, dtype=dtype)
            assert refused(1, fn, **{name: OnGpu(t), "dtype": given, ("row_stride" if name == "x" else "out_stride"): None}).startswith(name + " ")


def logprobs(**kw):
    a = dict(logits=FAKE, n_rows=3, vocab=96, targets=None, n_top=1, logprob=None, entropy=FAKE, top_ids=FAKE, top_logprobs=FAKE, ws=FAKE, dtype=sp.SP_LOGITS_F32,
             ws_bytes=1 << 30, stream=0)
    a.update(kw)
    sp.sp_logprobs(**a)


@pytest.mark.parametrize("fn,name,width", [(quantise, "x", 96), (matmul, "out", 5), (logprobs, "logits", 96)])
def test_rows_that_lie_on_top_of_one_another_are_refused(fn, name, width):
    """A row that was expanded holds one row's elements: no other stride may stand in for its 0, or rows behind it would be read or written."""
    import torch
    stride = "out_stride" if name == "out" else "row_stride"
    for dtype, kind in ((torch.float32, sp.SP_LOGITS_F32), (torch.bfloat16, sp.SP_LOGITS_BF16)):
        t = torch.zeros(1, width, dtype=dtype).expand(3, width)
        for given in (None, 0):
            assert "stride" in refused(1, fn, **{name: OnGpu(t), "dtype": kind, stride: given})
        refused(1, fn, **{name: OnGpu(t), "dtype": kind, stride: width})
    assert "stride" in refused(1, fn, **{stride: 0})


def test_host_tensors_are_refused():
    import torch
    refused(1, weights, q=torch.zeros(4, 8, 64, dtype=torch.bfloat16))
    refused(1, evict, k_pool=torch.zeros(4, 2, 64, 32, dtype=torch.uint8))
    refused(1, quantise, x=torch.zeros(3, 96, dtype=torch.bfloat16))
    refused(1, matmul, w_codes=torch.zeros(5, 48, dtype=torch.uint8))


@pytest.mark.parametrize("H,kv,d,offsets", [(32, 8, 64, [0, 1]), (32, 8, 64, [0, 8]), (16, 8, 128, [0, 1]), (16, 2, 128, [0, 3, 7]), (32, 8, 64, [0, 1, 513, 514])])
def test_attend_workspace_covers_shorter_contexts(H, kv, d, offsets):
    desc = cache(n_q_heads=H, n_kv_heads=kv, head_dim=d, stride_token=d, stride_head=64 * d, page_stride=kv * 64 * d, n_pages=1 << 20)
    off, most = sp.host_offsets(offsets), 0
    for n in [*range(1, 20000, 32), *(32 * (8 << 2 * e) + 32 * s + 1 for e in range(5, 11) for s in (-3, -2, -1, 0, 1, 2))]:
        size = sp.sp_attend_workspace(desc, off, len(offsets) - 1, n)
        assert size >= most, (n, size, most)
        most = size
    assert most > 0


@pytest.mark.parametrize("name", ["sp_weights.hip", "sp_evict.hip", "sp_mx4.hip"])
def test_files_that_may_meet_nans_are_compiled_to_honour_them(name):
    from paper_2603_02631_amd import build
    src = os.path.join(build.CSRC, name)
    assert src in build.sources()
    assert not [f for f in build.compile_command(src, "x.o") if "no-honor-nans" in f or "fast-math" in f or "finite-math" in f]


@pytest.mark.timeout(600)
def test_host_code_under_sanitizers(tmp_path):
    csrc = os.path.join(ROOT, "paper_2603_02631_amd", "csrc")
    srcs = [os.path.join(csrc, n) for n in ("sp_weights.hip", "sp_evict.hip", "sp_mx4.hip", "sp_cache.hip", "sp_attend.hip", "sp_common.cpp")]
    exe = str(tmp_path / "draft4_driver")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-fno-sanitize-recover=undefined",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "host", "draft4_driver.cpp"), *srcs, "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert run.returncode == 0, run.stdout[-4000:]
    assert "all checks passed" in run.stdout and "runtime error" not in run.stdout and "AddressSanitizer" not in run.stdout
