"""The few-rows kernel over a cache of 4 bits when its waits run out: a library whose waits give up at once (its copies are
waited for all the same) leaves the results as they were, raises the flag, and the device goes on."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_21858_gb300 import build, pps

pytestmark = pytest.mark.gpu

BF, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def impatient(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    pps.lib()
    build.build()
    d = str(tmp_path_factory.mktemp("impatient"))
    obj, so = os.path.join(d, "q4.o"), os.path.join(d, "libpps_impatient.so")
    subprocess.run([build.nvcc(), "-std=c++17", "-O3", "-Xcompiler", "-fPIC", "-I" + os.path.join(build.ROOT, "include"),
                    "-DPPS_WAIT_LIMIT=0", *build.ARCH, "-c", os.path.join(build.CSRC, "pps_attention_q4.cu"), "-o", obj], check=True)
    rest = [os.path.join(build.OUT, sub, src.replace(".cu", ".o"))
            for sub, sources in (("obj", build.SOURCES), ("obj_common", build.COMMON)) for src in sources if src != "pps_attention_q4.cu"]
    subprocess.run([build.nvcc(), *build.ARCH, "-shared", "-cudart", "static", "-o", so, obj, *rest], check=True)
    fn = ctypes.CDLL(so).pps_paged_attention_q4
    fn.argtypes, fn.restype = [ctypes.c_char_p, ctypes.c_void_p], ctypes.c_int
    return fn


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dt", [BF, F16])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("q_len,kv_len,heads,kv_heads,d", [([1, 1, 1], [900, 65, 3], 8, 2, 128), ([3, 1, 2], [70000, 10, 500], 16, 2, 128),
                                                           ([1] * 64, [2000 + i for i in range(64)], 8, 2, 128), ([2], [333], 4, 1, 64)])
def test_nothing_is_written_and_the_device_goes_on(impatient, q_len, kv_len, heads, kv_heads, d, layout, dt):
    g = torch.Generator(device="cuda").manual_seed(d + len(q_len))
    page, n, n_seq = 16, sum(q_len), len(q_len)
    assert n * heads // kv_heads <= 32 * n_seq  # (rows of the kernel in question)
    held = [-(-x // page) for x in kv_len]
    shape = (sum(held), kv_heads, page) if layout == "head" else (sum(held), page, kv_heads)

    def made(width, lo, hi):
        x = torch.randint(lo, hi, shape + (width,), generator=g, device="cuda", dtype=torch.uint8)
        return x.transpose(1, 2) if layout == "head" else x

    scales = pps.q4_scale_bytes(d)
    cache = pps.CacheQ4(made(d // 2, 0, 256), made(d // 2, 0, 256), made(scales, 40, 60), made(scales, 40, 60))
    pages = torch.zeros(n_seq, max(held), dtype=torch.int32, device="cuda")
    for s, h in enumerate(held):
        pages[s, :h] = i32(range(sum(held[:s]), sum(held[:s]) + h))
    lens, q_off = i32(kv_len), i32([sum(q_len[:s]) for s in range(n_seq + 1)])
    q = torch.randn(n, heads, d, generator=g, device="cuda").to(dt)
    want = pps.paged_attention_q4(q, cache, pages, lens, q_off)
    out, lse = torch.full_like(q, 7.0), torch.full((n, heads), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = pps.attention_q4_workspace(n, heads, kv_heads, d)
    k, ks = cache.k, cache.k_scale
    args = pps._ATTENTION_Q4_ARGS
    code = impatient(args.pack(args.size, q.data_ptr(), heads * d, d, out.data_ptr(), heads * d, d, k.data_ptr(), cache.v.data_ptr(),
                               ks.data_ptr(), cache.v_scale.data_ptr(), 0, 0, k.shape[0], page, kv_heads, d, *k.stride()[:3],
                               *ks.stride()[:3], pages.data_ptr(), lens.data_ptr(), q_off.data_ptr(), 0, lse.data_ptr(),
                               status.data_ptr(), ws.data_ptr(), ws.numel(), n, pages.shape[1], pps.BF16 if dt is BF else pps.F16,
                               heads, pages.shape[1], n_seq, 0, d ** -0.5),
                     torch.cuda.current_stream().cuda_stream)
    assert code == pps.OK
    torch.cuda.synchronize()
    assert int(status) == pps.FLAG_TIMEOUT
    assert bool((out == 7).all()) and bool((lse == 7).all())
    assert torch.equal(pps.paged_attention_q4(q, cache, pages, lens, q_off), want)
