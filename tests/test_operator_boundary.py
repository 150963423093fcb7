"""CPU-side checks of the cache, attention and log-probability entry points: bad host-visible arguments are refused with the
documented status before anything is launched (the addresses are fake and never dereferenced), calls without work are
no-ops, and the host code is clean under the address and undefined-behaviour sanitizers."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

import paper_2603_02631_amd as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FAKE = 0x10000


def cache(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, cache_type=sp.SP_CACHE_E4M3, n_pages=4, page_tokens=64,
                page_stride=2 * 64 * 64, stride_head=64 * 64, stride_token=64)
    base.update(kw)
    return sp.CacheDesc(*[base[f[0]] for f in sp.CacheDesc._fields_])


def refused(status, fn, *args, **kw):
    with pytest.raises(sp.SpError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value
    assert e.value.message


BAD_CACHES = [
    (dict(n_q_heads=0), 1), (dict(n_q_heads=7), 1), (dict(n_kv_heads=0), 1), (dict(n_kv_heads=-2), 1), (dict(cache_type=2), 1),
    (dict(n_pages=0), 1), (dict(n_pages=1 << 31), 1), (dict(page_tokens=0), 1), (dict(page_tokens=48), 1), (dict(page_tokens=1 << 25), 1),
    (dict(stride_token=48), 1), (dict(stride_token=72), 1), (dict(stride_token=-64), 1), (dict(stride_head=8), 1),
    (dict(stride_head=32), 1), (dict(page_stride=1 << 41), 1), (dict(page_stride=16), 1), (dict(page_stride=24), 1),
    (dict(head_dim=96), 2), (dict(head_dim=256), 2), (dict(n_q_heads=34), 2), (dict(n_q_heads=5000, n_kv_heads=5000), 2)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_cache_descriptions(kw, status):
    d = cache(**kw)
    refused(status, sp.sp_attend_workspace, d, [0, 1], 1, 64)
    refused(status, append, d)


def test_bf16_strides_are_multiples_of_eight():
    assert sp.sp_attend_workspace(cache(cache_type=sp.SP_CACHE_BF16, stride_token=72), [0, 1], 1, 64) >= 0
    refused(1, sp.sp_attend_workspace, cache(cache_type=sp.SP_CACHE_BF16, stride_token=68), [0, 1], 1, 64)


def append(d=None, **kw):
    a = dict(k=FAKE, v=FAKE, offsets_host=[0, 3], offsets_dev=FAKE, start=FAKE, block_table=FAKE, k_pool=FAKE, v_pool=FAKE,
             k_scale=FAKE, v_scale=FAKE, q=FAKE, q_out=FAKE, cos=FAKE, sin=FAKE, n_pos=100, rot_dim=64, rot_style=0, table_stride=4, stream=0)
    a.update(kw)
    sp.sp_cache_append(d or cache(), **a)


@pytest.mark.parametrize("kw", [
    dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(offsets_dev=None), dict(start=None), dict(block_table=None),
    dict(k_pool=None), dict(v_pool=None), dict(k_scale=None), dict(v_scale=None), dict(cos=None), dict(sin=None),
    dict(k=FAKE + 8), dict(v=FAKE + 2), dict(q=FAKE + 4), dict(q_out=FAKE + 8), dict(k_pool=FAKE + 8), dict(v_pool=FAKE + 4),
    dict(cos=FAKE + 4), dict(sin=FAKE + 8), dict(k_scale=FAKE + 2), dict(n_pos=0), dict(n_pos=-3),
    dict(rot_dim=8), dict(rot_dim=80), dict(rot_dim=-16), dict(rot_style=2), dict(table_stride=0), dict(k_stride=64), dict(v_stride=132),
    dict(q_stride=504), dict(k_stride=-128), dict(k_stride=1 << 41), dict(offsets_host=[1, 3]), dict(offsets_host=[0, 5, 3]),
    dict(offsets_host=[0, 1 << 31])])
def test_append_refuses(kw):
    refused(1, append, **kw)


def test_append_of_nothing_is_a_no_op():
    append(offsets_host=[0], k=None, v=None, q=None, q_out=None, offsets_dev=None)
    append(offsets_host=[0, 0, 0], k_pool=None)
    refused(1, append, offsets_host=[0] * 4098)


def attend(d=None, **kw):
    a = dict(q=FAKE, offsets_host=[0, 3, 4], offsets_dev=FAKE, lens=FAKE, max_len=200, block_table=FAKE, k_pool=FAKE, v_pool=FAKE,
             k_scale=FAKE, v_scale=FAKE, scale=0.125, out=FAKE, lse=FAKE, ws=FAKE, causal=1, window=0, table_stride=4,
             ws_bytes=1 << 40, stream=0)
    a.update(kw)
    sp.sp_attend(d or cache(), **a)


@pytest.mark.parametrize("kw", [
    dict(q=None), dict(out=None), dict(offsets_dev=None), dict(lens=None), dict(block_table=None), dict(k_pool=None), dict(v_pool=None),
    dict(k_scale=None), dict(v_scale=None), dict(q=FAKE + 8), dict(out=FAKE + 2), dict(k_pool=FAKE + 8), dict(v_scale=FAKE + 1),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(causal=-1), dict(window=-1),
    dict(causal=0, window=5), dict(max_len=257), dict(max_len=-1), dict(max_len=1 << 31, table_stride=1 << 30), dict(table_stride=0),
    dict(offsets_host=[0, 4, 3]), dict(offsets_host=[2, 3])])
def test_attend_refuses(kw):
    refused(1, attend, **kw)


def test_attend_workspace_rules():
    d = cache(n_pages=4096)
    n = sp.sp_attend_workspace(d, [0, 1], 1, 100000)
    assert n % 256 == 0
    if n:
        for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(ws_bytes=n - 1)):
            refused(3, attend, d, **{**dict(offsets_host=[0, 1], max_len=100000, table_stride=4096, ws_bytes=n), **kw})
    lib = sp.load_library()
    off = sp.host_offsets([0, 1])
    assert lib.sp_attend_workspace(ctypes.byref(d), off, 1, 64, None) == 1
    assert lib.sp_attend_workspace(None, off, 1, 64, ctypes.byref(ctypes.c_size_t())) == 1
    assert lib.sp_attend_workspace(ctypes.byref(d), None, 1, 64, ctypes.byref(ctypes.c_size_t())) == 1
    refused(1, sp.sp_attend_workspace, d, [0, 1], 2, 64)            # fewer offsets than requests
    refused(1, sp.sp_attend_workspace, d, [0] * 4098)


def test_attend_of_nothing_is_a_no_op():
    attend(offsets_host=[0], q=None, out=None, lens=None)
    attend(offsets_host=[0, 0], q=None, ws=None, ws_bytes=0)


def logprobs(**kw):
    a = dict(logits=FAKE, n_rows=2, vocab=100, targets=FAKE, n_top=3, logprob=FAKE, entropy=FAKE, top_ids=FAKE, top_logprobs=FAKE, ws=FAKE,
             dtype=sp.SP_LOGITS_F32, row_stride=100, ws_bytes=1 << 40, stream=0)
    a.update(kw)
    sp.sp_logprobs(**a)


@pytest.mark.parametrize("kw", [
    dict(logits=None), dict(targets=None), dict(logprob=None), dict(top_ids=None), dict(top_logprobs=None), dict(dtype=2), dict(dtype=-1),
    dict(n_rows=-1), dict(n_rows=1 << 31), dict(vocab=0), dict(vocab=1 << 31, row_stride=1 << 31), dict(n_top=-1), dict(n_top=33), dict(vocab=2, row_stride=2),
    dict(row_stride=99), dict(row_stride=1 << 41), dict(logits=FAKE + 2), dict(logits=FAKE + 1, dtype=sp.SP_LOGITS_BF16)])
def test_logprobs_refuses(kw):
    refused(1, logprobs, **kw)


def test_logprobs_workspace_rules_and_no_ops():
    n = sp.sp_logprobs_workspace(1, 200000, 32)
    assert n % 256 == 0
    if n:
        for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(ws_bytes=n - 1)):
            refused(3, logprobs, **{**dict(n_rows=1, vocab=200000, row_stride=200000, n_top=32, ws_bytes=n), **kw})
    logprobs(n_rows=0, logits=None, top_ids=None)
    assert sp.load_library().sp_logprobs_workspace(1, 10, 1, None) == 1


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    t = torch.zeros(4, 128, dtype=torch.bfloat16)
    refused(1, append, k=t)                                     # not a device tensor
    refused(1, attend, q=t)
    refused(1, logprobs, logits=torch.zeros(2, 100))
    refused(1, logprobs, dtype=None)                            # an address without a type


@pytest.mark.timeout(600)
def test_host_code_of_the_operators_under_sanitizers(tmp_path):
    csrc = os.path.join(ROOT, "paper_2603_02631_amd", "csrc")
    srcs = [os.path.join(csrc, n) for n in ("sp_cache.hip", "sp_attend.hip", "sp_logprobs.hip", "sp_common.cpp")]
    exe = str(tmp_path / "operator_driver")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-fno-sanitize-recover=undefined",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "host", "operator_driver.cpp"), *srcs, "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert run.returncode == 0, run.stdout[-4000:]
    assert "all checks passed" in run.stdout and "runtime error" not in run.stdout and "AddressSanitizer" not in run.stdout


@pytest.mark.parametrize("H,kv,d,offsets", [
    (32, 8, 64, [0, 1]), (32, 8, 64, [0, 8]), (32, 8, 64, [0, 16]), (16, 8, 128, [0, 1]), (16, 2, 128, [0, 3, 7]), (4, 4, 64, list(range(49))),
    (32, 8, 64, [0, 1, 513, 514])])
def test_attend_workspace_covers_shorter_contexts(H, kv, d, offsets):
    """A program sizes its workspace once, for the longest context, and calls with the lengths that it has reached."""
    desc = cache(n_q_heads=H, n_kv_heads=kv, head_dim=d, stride_token=d, stride_head=64 * d, page_stride=kv * 64 * d, n_pages=1 << 20)
    B, most, widest = len(offsets) - 1, 0, 0
    off = sp.host_offsets(offsets)
    # every length up to 20000 tokens that changes the number of blocks, then those around where a share's least number of blocks doubles
    lengths = list(range(1, 20000, 32)) + [32 * (8 << 2 * e) + 32 * s + 1 for e in range(5, 11) for s in (-3, -2, -1, 0, 1, 2)]
    for n in lengths:
        size = sp.sp_attend_workspace(desc, off, B, n)
        assert size >= most, (n, size, most, widest)
        if size > most:
            most, widest = size, n
    assert most > 0
    # what a call asks for is what the query says for its own length, and no more
    for n in (4064, 4065, 16346, 16384):
        size = sp.sp_attend_workspace(desc, off, B, n)
        kw = dict(offsets_host=offsets, max_len=n, table_stride=1 << 20)
        if size:
            refused(3, attend, desc, **kw, ws_bytes=size - 1)


@pytest.mark.parametrize("vocab", [4096, 32000, 50021, 128000, 262144])
@pytest.mark.parametrize("n_top", [0, 1, 32])
def test_logprobs_workspace_covers_fewer_rows(vocab, n_top):
    """A program sizes its workspace once, for the most rows; a call that needs none itself goes without."""
    sizes = [sp.sp_logprobs_workspace(n, vocab, n_top) for n in [*range(0, 600), 1000, 4096, (1 << 31) - 1]]
    assert sizes == sorted(sizes)
    if sizes[2]:
        refused(3, logprobs, n_rows=1, vocab=vocab, row_stride=vocab, n_top=n_top, ws_bytes=sizes[1] - 1)
        refused(3, logprobs, n_rows=2, vocab=vocab, row_stride=vocab, n_top=n_top, ws=None)


@pytest.mark.parametrize("name", ["sp_cache.hip", "sp_attend.hip"])
def test_files_that_may_meet_nans_are_compiled_to_honour_them(name):
    from paper_2603_02631_amd import build
    src = os.path.join(build.CSRC, name)
    assert src in build.sources()
    assert not [f for f in build.compile_command(src, "x.o") if "no-honor-nans" in f or "fast-math" in f or "finite-math" in f]


class OnGpu:
    """A tensor of the CPU that says it is on the GPU: the binding looks at it, the library refuses the call before anything is read."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)

    def data_ptr(self):
        return FAKE


INDEX_ARGUMENTS = [(append, "start", 2, 32), (append, "positions", 3, 32), (append, "block_table", 8, 32), (append, "offsets_dev", 3, 64),
                   (attend, "lens", 2, 32), (attend, "block_table", 8, 32), (attend, "offsets_dev", 3, 64),
                   (logprobs, "targets", 2, 32), (logprobs, "top_ids", 6, 32)]


@pytest.mark.parametrize("fn,name,n,bits", INDEX_ARGUMENTS)
def test_indices_of_another_width_are_refused(fn, name, n, bits):
    """64-bit integers are torch's own choice: read as 32-bit ones they would be every other one a zero."""
    import torch
    stop = {append: dict(rot_dim=8), attend: dict(causal=2), logprobs: dict(row_stride=1)}[fn]     # refused by the library in any case
    own, other = (torch.int32, torch.int64) if bits == 32 else (torch.int64, torch.int32)
    for dtype in (own, torch.uint32 if bits == 32 else torch.uint64):
        with pytest.raises(sp.SpError) as e:
            fn(**{name: OnGpu(torch.zeros(2 * n, dtype=dtype)), **stop})
        assert name not in e.value.message, e.value
    for dtype in (other, torch.float32, torch.float64, torch.int16):
        with pytest.raises(sp.SpError) as e:
            fn(**{name: OnGpu(torch.zeros(4 * n, dtype=dtype)), **stop})
        assert e.value.status == 1 and name in e.value.message, e.value


@pytest.mark.parametrize("fn,name,shape,own", [
    (append, "k", (3, 128), "bfloat16"), (append, "v", (3, 128), "bfloat16"), (append, "q", (3, 512), "bfloat16"), (append, "q_out", (3, 512), "bfloat16"),
    (append, "k", (3, 2, 64), "bfloat16"), (append, "q", (3, 8, 64), "bfloat16"),
    (append, "cos", (100, 32), "float32"), (append, "sin", (100, 32), "float32"), (append, "k_scale", (4, 2, 2), "float32"), (append, "v_scale", (4, 2, 2), "float32"),
    (append, "k_pool", (4, 2, 64, 64), "float8_e4m3fn"), (append, "v_pool", (4, 2, 64, 64), "float8_e4m3fn"),
    (attend, "q", (4, 8, 64), "bfloat16"), (attend, "out", (4, 8, 64), "bfloat16"), (attend, "lse", (4, 8), "float32"), (attend, "k_scale", (4, 2, 2), "float32"),
    (attend, "v_scale", (4, 2, 2), "float32"), (attend, "k_pool", (4, 2, 64, 64), "float8_e4m3fn"), (attend, "v_pool", (4, 2, 64, 64), "float8_e4m3fn"),
    (logprobs, "logprob", (2,), "float32"), (logprobs, "entropy", (2,), "float32"), (logprobs, "top_logprobs", (2, 3), "float32")])
def test_numbers_of_another_type_are_refused(fn, name, shape, own):
    """float16 has bf16's width and float64 more than enough bytes: both would be misread without a word. Integers of an element's width are its bits."""
    import torch
    stop = {append: dict(rot_dim=8, offsets_host=[0, 2, 3]), attend: dict(causal=2), logprobs: dict(row_stride=1)}[fn]
    bits = {"bfloat16": ("int16",), "float32": ("int32",), "float8_e4m3fn": ("uint8", "int8")}[own]
    for dtype in (own, *bits):
        with pytest.raises(sp.SpError) as e:
            fn(**{name: OnGpu(torch.zeros(shape, dtype=getattr(torch, dtype))), **stop})
        assert not e.value.message.startswith(name + " "), e.value
    others = {"bfloat16": ("float16", "float32", "float64"), "float32": ("float64",), "float8_e4m3fn": ("float8_e5m2", "float16", "float32")}[own]
    for dtype in others:
        with pytest.raises(sp.SpError) as e:
            fn(**{name: OnGpu(torch.zeros(shape, dtype=getattr(torch, dtype))), **stop})
        assert e.value.status == 1 and e.value.message.startswith(name + " "), e.value


def test_pools_of_a_bf16_cache_are_of_its_type():
    import torch
    d = cache(cache_type=sp.SP_CACHE_BF16)
    for dtype in (torch.bfloat16, torch.int16, torch.uint16):
        refused_by_library = dict(k_pool=OnGpu(torch.zeros(4, 2, 64, 64, dtype=dtype)))
        with pytest.raises(sp.SpError) as e:
            attend(d, causal=2, **refused_by_library)
        assert "causal" in e.value.message
    for dtype in (torch.float16, torch.float32):
        with pytest.raises(sp.SpError) as e:
            attend(d, causal=2, k_pool=OnGpu(torch.zeros(4, 2, 64, 64, dtype=dtype)))
        assert e.value.message.startswith("k_pool ")


@pytest.mark.parametrize("given", [None, sp.SP_LOGITS_BF16, sp.SP_LOGITS_F32])
def test_logits_of_another_type_are_refused(given):
    """A projection's output in float16 gave likely-looking tokens and probabilities of its bits read as bf16."""
    import torch
    for dtype, own in ((torch.bfloat16, sp.SP_LOGITS_BF16), (torch.int16, sp.SP_LOGITS_BF16), (torch.float32, sp.SP_LOGITS_F32),
                       (torch.int32, sp.SP_LOGITS_F32), (torch.float16, -1), (torch.float64, -1), (torch.int64, -1)):
        for shape in ((2, 100), (2, 1, 100)):
            with pytest.raises(sp.SpError) as e:
                logprobs(logits=OnGpu(torch.zeros(shape, dtype=dtype)), dtype=given, row_stride=None, n_top=33)
            fits = own >= 0 and given in (None, own)
            assert ("n_top" in e.value.message) == fits and e.value.message.startswith("logits ") == (not fits), (dtype, e.value)


def test_attend_scales_stay_finite_in_units_of_log_2():
    for scale in (2.3e38, 1.0, 1e-38):
        with pytest.raises(sp.SpError) as e:
            attend(scale=scale, causal=2)
        assert "causal" in e.value.message
    for scale in (2.4e38, 2.9e38, 3.4e38):
        with pytest.raises(sp.SpError) as e:
            attend(scale=scale, causal=2)
        assert "scale" in e.value.message
