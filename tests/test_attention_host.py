"""The attention half of a layer, host side: sizes, frequencies, and every refusal (they come before the first HIP call, so they
run without a GPU)."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2603_27914_amd import binding, build

    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    return binding.lib()


def test_cache_sizes(L):
    assert L.itq3s_cache_bytes(1, 32, 1, 128) == 32 * 132
    assert L.itq3s_cache_bytes(7, 256, 8, 64) == 7 * 8 * 8 * (32 * 64 + 128)
    assert L.itq3s_cache_bytes(2**22, 1024, 8, 256) == 2**22 * 8 * 32 * (32 * 256 + 128)
    assert L.itq3s_cache_bytes(2**31 - 1, 65536, 1024, 256) == 0  # beyond 2^48 bytes
    for bad in ((0, 32, 1, 64), (1, 16, 1, 64), (1, 48, 1, 64), (1, 131072, 1, 64), (1, 32, 0, 64), (1, 32, 1025, 64), (1, 32, 1, 96), (2**31, 32, 1, 64), (-1, 32, 1, 64)):
        assert L.itq3s_cache_bytes(*bad) == 0


def test_workspace_sizes(L):
    ws = L.itq3s_cache_attention_workspace_bytes
    assert ws(1, 1, 8, 1, 128, 1, 32) == 256                                     # one part: nothing to park
    assert ws(1, 1, 64, 8, 128, 1, 131072) >= 2 * 64 * 130 * 4                   # several
    assert ws(4, 1, 8, 2, 64, 10**9, 100) == ws(4, 1, 8, 2, 64, 4, 100)          # no sequence has more rows than there are
    for bad in ((0, 1, 8, 2, 64, 1, 1), (1, 0, 8, 2, 64, 1, 1), (1, 1, 9, 2, 64, 1, 1), (1, 1, 8, 2, 65, 1, 1), (1, 1, 8, 2, 64, 0, 1), (1, 1, 8, 2, 64, 1, 0)):
        assert ws(*bad) == 256


def test_rope_frequencies(L):
    from paper_2603_27914_amd import binding

    for rot, base in ((128, 10000.0), (64, 500000.0), (2, 1.0), (256, 1e6)):
        want = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
        assert np.allclose(binding.itq3s_rope_frequencies(rot, base).numpy(), want, rtol=1e-15)
        assert np.allclose(binding.itq3s_rope_frequencies(rot, base, 8.0).numpy(), np.array(want) / 8.0, rtol=1e-15)
    f = binding.itq3s_rope_frequencies(128, 500000.0, 8.0, 8192, 1.0, 4.0).numpy()
    g = binding.itq3s_rope_frequencies(128, 500000.0).numpy()
    turns = 8192 * g / (2 * math.pi)
    assert np.array_equal(f[turns >= 4.0], g[turns >= 4.0]) and np.allclose(f[turns <= 1.0], g[turns <= 1.0] / 8, rtol=1e-15)
    mid = (turns > 1.0) & (turns < 4.0)
    share = (turns[mid] - 1) / 3
    assert mid.any() and np.allclose(f[mid], share * g[mid] + (1 - share) * g[mid] / 8, rtol=1e-14)
    out = (ctypes.c_double * 128)()
    for bad in ((0, 1e4, 1.0, 0, 1.0, 4.0), (3, 1e4, 1.0, 0, 1.0, 4.0), (258, 1e4, 1.0, 0, 1.0, 4.0), (64, 0.0, 1.0, 0, 1.0, 4.0), (64, 1e4, 0.0, 0, 1.0, 4.0), (64, float("nan"), 1.0, 0, 1.0, 4.0),
                (64, 1e4, float("inf"), 0, 1.0, 4.0), (64, 1e4, 2.0, -1, 1.0, 4.0), (64, 1e4, 2.0, 100, 4.0, 4.0), (64, 1e4, 2.0, 100, -1.0, 4.0)):
        assert L.itq3s_rope_frequencies(*bad, out) == -2
    assert L.itq3s_rope_frequencies(64, 1e4, 1.0, 0, 1.0, 4.0, None) == -1
    with pytest.raises(binding.Itq3sError):
        binding.itq3s_rope_frequencies(7)


class Call:
    """A call's arguments by name, each to be replaced."""

    def __init__(self, f, **args):
        self.f, self.args = f, args

    def __call__(self, **other):
        assert set(other) <= set(self.args)
        return self.f(*{**self.args, **other}.values())


@pytest.fixture(scope="module")
def memory():
    buf = (ctypes.c_uint8 * 8192)()
    at = (ctypes.addressof(buf) + 255) & ~255
    return buf, ctypes.c_void_p(at), ctypes.c_void_p(at + 8), ctypes.c_void_p(at + 2)


class CacheDesc(ctypes.Structure):
    """struct itq3s_cache"""

    _fields_ = [("data", ctypes.c_void_p), ("pages", ctypes.c_int64), ("page_tokens", ctypes.c_int), ("kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int)]


def desc(data, pages=1, page_tokens=32, kv_heads=2, head_dim=64):
    return ctypes.pointer(CacheDesc(data.value if data is not None else None, pages, page_tokens, kv_heads, head_dim))


def test_the_binding_packs_the_descriptor_as_c_does():
    import torch

    from paper_2603_27914_amd import binding

    data = torch.zeros(3 * 5 * 2 * (32 * 64 + 128), dtype=torch.uint8)
    packed = binding._need_cache(binding.Cache(data, 64, 5, 64))
    d = CacheDesc.from_buffer_copy(packed)
    assert len(packed) == ctypes.sizeof(CacheDesc) and (d.data, d.pages, d.page_tokens, d.kv_heads, d.head_dim) == (data.data_ptr(), 3, 64, 5, 64)


def test_append_refuses(L, memory):
    _, ok, by8, by2 = memory
    c = Call(L.itq3s_cache_append, Q=ok, ldq=512, q_heads=8, K=ok, ldk=128, V=ok, ldv=128, T=1, in_dtype=1, kv_heads=2, head_dim=64, q_norm=ok, k_norm=ok, eps=1e-6, positions=ok, freq=ok, rot=64,
             interleaved=0, gain=1.0, Q_out=ok, ldqo=512, K_out=ok, ldko=128, out_dtype=1, cache=desc(ok), slots=ok, flags=None, stream=None)
    for n in ("K", "V", "slots", "positions", "freq", "Q_out"):
        assert c(**{n: None}) == -1, n
    assert c(cache=None) == -1                                    # V without a cache
    assert c(cache=None, V=None, K_out=None) == -1                # rotated keys to nowhere
    assert c(cache=None, V=None, Q=None, K=None) == -1
    assert c(cache=desc(None)) == -1
    for other in (dict(T=0), dict(T=2**31), dict(head_dim=96), dict(head_dim=128), dict(kv_heads=1), dict(kv_heads=0), dict(q_heads=0), dict(rot=72), dict(rot=80), dict(rot=-16), dict(rot=8), dict(eps=-1.0),
                  dict(eps=float("nan")), dict(gain=float("inf")), dict(ldq=504), dict(ldk=120), dict(ldv=120), dict(ldqo=504), dict(ldko=120), dict(cache=desc(ok, page_tokens=48)),
                  dict(cache=desc(ok, pages=0)), dict(cache=desc(ok, head_dim=128))):
        assert c(**other) == -2, other
    for other in (dict(Q=by8), dict(K=by8), dict(V=by2), dict(Q_out=by8), dict(K_out=by8), dict(ldq=516), dict(ldk=132), dict(ldv=130), dict(ldqo=516), dict(ldko=132), dict(q_norm=by8), dict(k_norm=by2),
                  dict(positions=by2), dict(freq=by2), dict(slots=by2), dict(cache=desc(by8)), dict(flags=by2)):
        assert c(**other) == -3, other
    assert c(in_dtype=2) == -4 and c(out_dtype=-1) == -4


def test_read_refuses(L, memory):
    _, ok, by8, by2 = memory
    c = Call(L.itq3s_cache_read, cache=desc(ok), slots=ok, T=1, K=ok, ldk=128, V=ok, ldv=128, out_dtype=0, flags=None, stream=None)
    for n in ("cache", "slots", "K", "V"):
        assert c(**{n: None}) == -1
    for other in (dict(T=0), dict(T=2**31), dict(ldk=127), dict(ldv=64), dict(cache=desc(ok, kv_heads=0))):
        assert c(**other) == -2
    for other in (dict(K=by8), dict(V=by2), dict(ldk=130), dict(ldv=129), dict(slots=by2), dict(flags=by2), dict(cache=desc(by2))):
        assert c(**other) == -3
    assert c(out_dtype=5) == -4


def test_cache_attention_refuses(L, memory):
    _, ok, by8, by2 = memory
    c = Call(L.itq3s_cache_attention, Q=ok, ldq=512, T=1, q_heads=8, cache=desc(ok), q_starts=ok, kv_lens=ok, seqs=1, pages=ok, ld_pages=1, max_q=1, max_kv=32, scale=0.1, out=ok, ldo=512, workspace=ok,
             workspace_bytes=256, flags=None, stream=None)
    for n in ("Q", "cache", "q_starts", "kv_lens", "pages", "out"):
        assert c(**{n: None}) == -1
    for other in (dict(T=0), dict(T=2**30), dict(q_heads=7), dict(q_heads=0), dict(seqs=0), dict(seqs=2**24 + 1), dict(ld_pages=0), dict(ld_pages=2**30), dict(max_q=0), dict(max_kv=0), dict(max_kv=2**31),
                  dict(scale=float("nan")), dict(ldq=256), dict(ldo=256), dict(cache=desc(ok, head_dim=32))):
        assert c(**other) == -2, other
    for other in (dict(Q=by8), dict(out=by8), dict(ldq=516), dict(ldo=516), dict(q_starts=by2), dict(kv_lens=by2), dict(pages=by2), dict(flags=by2), dict(workspace=by8)):
        assert c(**other) == -3, other
    assert c(workspace=None) == -5 and c(workspace_bytes=255) == -5 and c(ld_pages=1000, max_kv=32000, workspace_bytes=4096) == -5


def test_prompt_attention_refuses(L, memory):
    _, ok, by8, by2 = memory
    c = Call(L.itq3s_prompt_attention, Q=ok, ldq=512, K=ok, ldk=128, V=ok, ldv=128, T=1, q_heads=8, kv_heads=2, head_dim=64, starts=ok, seqs=1, max_len=1, causal=1, scale=0.1, out=ok, ldo=512, stream=None)
    for n in ("Q", "K", "V", "starts", "out"):
        assert c(**{n: None}) == -1
    for other in (dict(T=0), dict(T=2**29), dict(q_heads=9), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=80), dict(seqs=0), dict(max_len=0), dict(scale=float("inf")), dict(ldq=511), dict(ldk=64),
                  dict(ldv=64), dict(ldo=64)):
        assert c(**other) == -2, other
    for other in (dict(Q=by8), dict(K=by2), dict(V=by8), dict(out=by8), dict(ldq=516), dict(ldk=130), dict(ldv=132), dict(ldo=514), dict(starts=by2)):
        assert c(**other) == -3, other


def test_sizes_beyond_a_launch_are_refused(L, memory):
    """A launch has less than 2^32 threads."""
    _, ok, _, _ = memory
    wide = desc(ok, kv_heads=1024)
    assert L.itq3s_cache_append(None, 0, 0, ok, 128, ok, 128, 2**24 + 1, 1, 2, 64, None, None, 0.0, None, None, 0, 0, 1.0, None, 0, None, 0, 1, desc(ok), ok, None, None) == -2
    assert L.itq3s_cache_read(desc(ok), ok, 2**28 + 1, ok, 128, ok, 128, 0, None, None) == -2
    assert L.itq3s_cache_attention(ok, 65536, 1, 1024, wide, ok, ok, 4097, ok, 1, 1, 32, 0.1, ok, 65536, ok, 4096, None, None) == -2
    assert L.itq3s_prompt_attention(ok, 65536, ok, 65536, ok, 65536, 1, 1024, 1024, 64, ok, 4097, 1, 1, 0.1, ok, 65536, None) == -2


def test_binding_refuses_what_the_library_cannot_see(monkeypatch):
    """Pointers carry neither sizes nor types: those are checked before the call (here on CPU tensors that pass for device ones, with a library that is
    not to be reached)."""
    import torch

    from paper_2603_27914_amd import binding

    monkeypatch.setattr(binding, "_need_here", lambda *t: None)
    monkeypatch.setattr(binding, "_check", lambda status: pytest.fail("the library was called"))
    monkeypatch.setattr(binding, "_stream", lambda: pytest.fail("the library was called"))
    E = binding.Itq3sError
    h, f, i32, i64, f64 = torch.float16, torch.float32, torch.int32, torch.int64, torch.float64
    cache = binding.Cache(torch.zeros(2 * 2 * 2176, dtype=torch.uint8), 32, 2, 64)
    assert cache.pages == 2
    q, k = torch.zeros((3, 512), dtype=h), torch.zeros((3, 128), dtype=h)
    pos, slots, freq = torch.zeros(3, dtype=i32), torch.zeros(3, dtype=i64), torch.zeros(32, dtype=f64)
    good = dict(q=q, k=k, v=k, positions=pos, freq=freq, cache=cache, slots=slots)
    for other in (dict(q=q.float()), dict(q=q[:2]), dict(q=q[:, :500]), dict(q=torch.zeros((3, 1024), dtype=h)[:, ::2]), dict(k=k[:, :64]), dict(k=k.float()), dict(v=k[:2]), dict(v=None), dict(k=None), dict(slots=None),
                  dict(slots=pos), dict(slots=slots[:2]), dict(positions=None), dict(positions=slots), dict(positions=pos[:1]), dict(freq=freq.float()), dict(freq=torch.zeros((2, 16), dtype=f64)),
                  dict(q_norm=torch.zeros(64, dtype=h)), dict(k_norm=torch.zeros(128, dtype=f)), dict(q_out=q[:, :64]), dict(q_out=torch.zeros((3, 512), dtype=f), k_out=k.clone()), dict(k_out=k[:2]),
                  dict(status_flags=torch.zeros(1)), dict(cache=cache._replace(data=cache.data[:-1])), dict(cache=cache._replace(page_tokens=48)), dict(cache=cache._replace(data=cache.data.view(i32))),
                  dict(cache=None), dict(cache=None, v=None), dict(cache=None, v=None, head_dim=63), dict(q=None, k=None), dict(q=None, q_out=q)):
        with pytest.raises(E):
            binding.itq3s_cache_append(**{**good, **other})
    for args in (dict(slots=pos), dict(slots=slots[None]), dict(k_out=k.double()), dict(k_out=k, v_out=k.float()), dict(v_out=k[:, :64])):
        with pytest.raises(E):
            binding.itq3s_cache_read(cache, **{"slots": slots, **args})
    good = dict(q=q, cache=cache, q_starts=torch.zeros(3, dtype=i32), kv_lens=torch.zeros(2, dtype=i32), pages=torch.zeros((2, 4), dtype=i32))
    for other in (dict(q=q.float()), dict(q=q[0]), dict(q=q[:, :100]), dict(q_starts=torch.zeros(2, dtype=i32)), dict(q_starts=torch.zeros(3, dtype=i64)), dict(kv_lens=torch.zeros(3, dtype=i32)), dict(kv_lens=torch.zeros((2, 1), dtype=i32)),
                  dict(pages=torch.zeros((1, 4), dtype=i32)), dict(pages=torch.zeros(8, dtype=i32)), dict(pages=torch.zeros((2, 8), dtype=i32)[:, :4]), dict(pages=torch.zeros((2, 4), dtype=i64)),
                  dict(pages=torch.zeros((2, 0), dtype=i32)), dict(out=q.float()), dict(out=q[:2]), dict(workspace=torch.zeros(4096)), dict(status_flags=torch.zeros(1))):
        with pytest.raises(E):
            binding.itq3s_cache_attention(**{**good, **other})
    good = dict(q=q, k=k, v=k, head_dim=64, starts=torch.zeros(2, dtype=i32))
    for other in (dict(q=q.float()), dict(k=k.float()), dict(v=k[:2]), dict(v=k[:, :64]), dict(head_dim=65), dict(k=k[:, :100]), dict(starts=torch.zeros(1, dtype=i32)), dict(starts=torch.zeros(2, dtype=i64)), dict(out=q.float()), dict(q=q[0])):
        with pytest.raises(E):
            binding.itq3s_prompt_attention(**{**good, **other})


def test_binding_keeps_to_the_current_device(monkeypatch):
    from paper_2603_27914_amd import binding

    class Tensor:
        def __init__(self, index):
            self.index, self.is_cuda = index, index >= 0

        def get_device(self):
            return self.index

    monkeypatch.setattr(binding, "_device", lambda: 1)
    binding._need_here(Tensor(1), None, Tensor(1))
    for tensors in ((Tensor(0),), (Tensor(1), Tensor(0)), (Tensor(-1),), (Tensor(1), None, Tensor(-1))):
        with pytest.raises(binding.Itq3sError):
            binding._need_here(*tensors)


@pytest.mark.parametrize("source", ["cache", "cache_attn", "prompt"])
def test_attention_kernels_keep_their_registers(source):
    from paper_2603_27914_amd import build

    src = os.path.join(build.CSRC, "itq3s_%s.hip" % source)
    asm = subprocess.run(["hipcc", *build.flags(src), "--cuda-device-only", "-S", src, "-o", "-"], check=True, stdout=subprocess.PIPE, stderr=subprocess.DEVNULL, text=True).stdout
    kernels = re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", asm, flags=re.S)
    assert kernels and [k for k in kernels if k[1] != "0"] == []
    # the copies written in assembly set m0, which cannot be named as clobbered: where there are any, nothing else uses it
    written, other = [], []
    for block in re.split(r"(;;?#ASMSTART.*?;;?#ASMEND)", asm, flags=re.S):
        (written if block.lstrip(";").startswith("#ASMSTART") else other).append(block)
    copies = [w for w in written if re.search(r"\bm0\b", w)]
    assert bool(copies) == (source == "prompt")
    assert not copies or not any(re.search(r"^\s+\w.*\bm0\b", o, flags=re.M) for o in other)
