"""The attention half of a decoder layer, without a GPU: refusals of the C entry points and of the binding, size queries, how a ragged
batch is dealt out (compiled for the host), the plain forms the GPU tests compare with."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

import __graft_entry__ as entry
import kv_ref as R
from paper_2307_09782_b200 import attention_fp8, binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, ALIGN, MODE, WORKSPACE = -1, -2, -3, -4, -5
P = 1 << 20  # an aligned address that nothing reads: every call here ends before a launch


@pytest.fixture(scope="module")
def L():
    entry.build()
    return binding.lib()


NORM = dict(q=P, ldq=1024, Hq=8, k=P, ldk=1024, H=2, T=5, D=128, wq=P, wk=P, eps=1e-6, table=P, far=100, rot=128, pairs=0, positions=P,
            qo=P, ldqo=1024, ko=P, ldko=256, stream=None)
BACK = dict(dq=P, lddq=1024, dk=P, lddk=256, q=P, ldq=1024, Hq=8, k=P, ldk=1024, H=2, T=5, D=128, wq=P, wk=P, eps=1e-6, table=P,
            far=100, rot=128, pairs=0, positions=P, dxq=P, lddxq=1024, dxk=P, lddxk=256, dwq=P, dwk=P, ws=P, bytes=1 << 30, stream=None)
WRITE = dict(k=P, ldk=256, v=P, ldv=256, T=5, cu=P, B=3, lens=P, table=P, table_ld=7, codes=P, scale=P, pages=9, H=2, page=64, D=128,
             mode=0, stream=None)
READ = dict(codes=P, scale=P, pages=9, H=2, page=64, D=128, table=P, table_ld=7, cu=P, B=3, T=5, k=P, v=P, dt=1, stream=None)
ATTN = dict(q=P, ldq=1024, Hq=8, T=5, cu=P, B=3, lens=P, table=P, table_ld=7, codes=P, scale=P, pages=9, H=2, page=64, D=128,
            sm=0.1, causal=1, window=0, out=P, dt=1, ldo=1024, lse=None, ws=P, bytes=1 << 30, stream=None)
CALLS = {"zq_qk_norm_rope": NORM, "zq_qk_norm_rope_backward": BACK, "zq_kv_cache_write": WRITE, "zq_kv_cache_read": READ,
         "zq_kv_attention": ATTN}
CACHE = [(dict(page=48), SHAPE), (dict(page=256), SHAPE), (dict(D=96), SHAPE), (dict(pages=0), SHAPE), (dict(H=0), SHAPE),
         (dict(pages=1 << 30, H=2), SHAPE), (dict(B=-1), SHAPE), (dict(T=-1), SHAPE), (dict(T=1 << 31), SHAPE),
         (dict(table_ld=-1), SHAPE), (dict(codes=None), NULL), (dict(scale=None), NULL), (dict(table=None), NULL),
         (dict(codes=P + 8), ALIGN), (dict(scale=P + 2), ALIGN), (dict(table=P + 1), ALIGN), (dict(cu=P + 2), ALIGN)]
ROPE = [(dict(D=96), SHAPE), (dict(D=256), SHAPE), (dict(rot=0), SHAPE), (dict(rot=24), SHAPE), (dict(rot=144), SHAPE),
        (dict(D=64, rot=128), SHAPE), (dict(far=0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=math.nan), SHAPE), (dict(eps=math.inf), SHAPE),
        (dict(pairs=2), MODE), (dict(T=-1), SHAPE), (dict(Hq=-1), SHAPE), (dict(ldq=1016), SHAPE), (dict(wq=None), NULL),
        (dict(table=None), NULL), (dict(positions=None), NULL), (dict(q=P + 8), ALIGN), (dict(ldk=1028), ALIGN),
        (dict(table=P + 4), ALIGN), (dict(wk=P + 4), ALIGN), (dict(positions=P + 2), ALIGN), (dict(H=70000), SHAPE)]
REFUSALS = {
    "zq_qk_norm_rope": ROPE + [(dict(ldqo=8), SHAPE), (dict(qo=None), NULL), (dict(ko=P + 2), ALIGN), (dict(ldko=260), ALIGN)],
    "zq_qk_norm_rope_backward": ROPE + [(dict(lddq=8), SHAPE), (dict(dq=None), NULL), (dict(dwq=None), NULL), (dict(dxk=None), NULL),
                                        (dict(q=None), NULL), (dict(dwk=P + 2), ALIGN), (dict(lddk=260), ALIGN), (dict(ws=None), WORKSPACE),
                                        (dict(bytes=1000), WORKSPACE), (dict(ws=P + 16), ALIGN)],
    "zq_kv_cache_write": CACHE + [(dict(lens=None), NULL), (dict(lens=P + 2), ALIGN), (dict(cu=None), SHAPE), (dict(mode=2), MODE),
                                  (dict(mode=16), MODE), (dict(ldk=128), SHAPE), (dict(ldv=260), ALIGN), (dict(k=None), NULL), (dict(v=P + 4), ALIGN)],
    "zq_kv_cache_read": CACHE + [(dict(cu=None), NULL), (dict(dt=2), MODE), (dict(k=None), NULL), (dict(v=P + 8), ALIGN)],
    "zq_kv_attention": CACHE + [(dict(lens=None), NULL), (dict(lens=P + 2), ALIGN), (dict(cu=None), SHAPE), (dict(dt=3), MODE),
                                (dict(causal=2), MODE), (dict(causal=0, window=4), MODE), (dict(window=-1), SHAPE), (dict(sm=0.0), SHAPE),
                                (dict(sm=-1.0), SHAPE), (dict(sm=math.nan), SHAPE), (dict(sm=math.inf), SHAPE), (dict(Hq=7), SHAPE),
                                (dict(Hq=0), SHAPE), (dict(ldq=8), SHAPE), (dict(ldo=8), SHAPE), (dict(q=None), NULL), (dict(out=None), NULL),
                                (dict(q=P + 8), ALIGN), (dict(ldq=1028), ALIGN), (dict(ldo=1028), ALIGN), (dict(out=P + 2), ALIGN),
                                (dict(lse=P + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(bytes=4096), WORKSPACE), (dict(ws=P + 64), ALIGN),
                                (dict(T=1 << 30, H=1), SHAPE)],
}


@pytest.mark.parametrize("name", list(CALLS))
def test_refusals(L, name):
    for change, status in REFUSALS[name]:
        assert set(change) <= set(CALLS[name]), change
        assert getattr(L, name)(*{**CALLS[name], **change}.values()) == status, (name, change)


@pytest.mark.parametrize("name", list(CALLS))
def test_nothing_to_do(L, name):
    change = dict(T=0, B=0) if "B" in CALLS[name] else dict(T=0)
    if name == "zq_qk_norm_rope_backward":
        change.update(wq=None, wk=None)
    assert getattr(L, name)(*{**CALLS[name], **change}.values()) == 0


def test_size_queries(L):
    assert binding.qk_norm_rope_backward_workspace_bytes(96) == 0
    assert binding.qk_norm_rope_backward_workspace_bytes(128) == 2 * binding.qk_norm_rope_backward_workspace_bytes(64) - (256 + 65536 + 37632)
    one = binding.kv_attention_workspace_bytes(1, 1, 8, 2, 128)
    assert one >= 148 * 256 * 130 * 4
    for wrong in ((-1, 1, 8, 2, 128), (1, -1, 8, 2, 128), (1, 1, 7, 2, 128), (1, 1, 8, 0, 128), (1, 1, 8, 2, 96), (1, 1, 0, 2, 64)):
        assert binding.kv_attention_workspace_bytes(*wrong) == 0
    sizes = [binding.kv_attention_workspace_bytes(T, B, 8, 2, 128) for T, B in ((0, 0), (64, 64), (4096, 1000000), (1 << 20, 1 << 30))]
    assert sizes == sorted(sizes)


def tensors(T=5, Hq=8, H=2, D=128, page=64):
    return (torch.zeros((T, Hq, D), dtype=torch.bfloat16), torch.zeros((T, H, D), dtype=torch.bfloat16),
            binding.make_kv_cache(9, H, D, page, "cpu"), torch.zeros((T, 7), dtype=torch.int32), torch.zeros(T, dtype=torch.int32))


def test_binding_refuses_what_it_cannot_describe(L):
    q, k, cache, pages, lens = tensors()
    rope = torch.zeros((10, 128))
    host = "CUDA tensor"
    bad = [
        (host, lambda: binding.qk_norm_rope(q, k, rope, lens)),
        ("bf16 tensor", lambda: binding.qk_norm_rope(q.float(), k, rope, lens)),
        ("side by side", lambda: binding.qk_norm_rope(q[:, ::2], k, rope, lens)),
        ("side by side", lambda: binding.qk_norm_rope(q[..., ::2], k[..., ::2], rope, lens)),
        ("belong together", lambda: binding.qk_norm_rope(q[:4], k, rope, lens)),
        ("positions", lambda: binding.qk_norm_rope(q, k, rope, lens.long())),
        ("positions", lambda: binding.qk_norm_rope(q, k, rope, lens[:4].contiguous())),
        ("table", lambda: binding.qk_norm_rope(q, k, rope.double(), lens)),
        ("both norms", lambda: binding.qk_norm_rope(q, k, rope, lens, wq=torch.ones(128))),
        ("wq", lambda: binding.qk_norm_rope(q, k, rope, lens, wq=torch.ones(64), wk=torch.ones(64))),
        ("gradients", lambda: binding.qk_norm_rope_backward(q[:, :4], k, q, k, rope, lens)),
        (host, lambda: binding.kv_cache_write(cache, k, k, pages, lens)),
        ("do not fit", lambda: binding.kv_cache_write(cache, q, q, pages, lens)),
        ("do not fit", lambda: binding.kv_cache_write(cache, k, q, pages, lens)),
        ("without cu", lambda: binding.kv_cache_write(cache, k[:4], k[:4], pages, lens)),
        ("cu", lambda: binding.kv_cache_write(cache, k, k, pages, lens, cu=lens)),
        ("lens", lambda: binding.kv_cache_write(cache, k, k, pages, lens.long())),
        ("table", lambda: binding.kv_cache_write(cache, k, k, pages[0], lens)),
        ("table", lambda: binding.kv_cache_write(cache, k, k, pages.t(), lens)),
        (host, lambda: binding.kv_cache_read(cache, pages, torch.zeros(6, dtype=torch.int32), 5)),
        ("out_dtype", lambda: binding.kv_cache_read(cache, pages, torch.zeros(6, dtype=torch.int32), 5, out_dtype=torch.float16)),
        ("cu", lambda: binding.kv_cache_read(cache, pages, None, 5)),
        (host, lambda: binding.kv_attention(cache, q, pages, lens)),
        ("does not fit", lambda: binding.kv_attention(cache, q[:, :7], pages, lens)),
        ("does not fit", lambda: binding.kv_attention(cache, torch.zeros((5, 8, 64), dtype=torch.bfloat16), pages, lens)),
        ("out_dtype", lambda: binding.kv_attention(cache, q, pages, lens, out_dtype=torch.float8_e4m3fn)),
        ("pages of", lambda: binding.make_kv_cache(2, 2, 128, 48, "cpu")),
        ("heads of", lambda: binding.make_kv_cache(2, 2, 80, 64, "cpu")),
        ("scales", lambda: binding.Fp8KvCache(cache.codes, cache.scale[:, :, :1])),
        ("contiguous", lambda: binding.Fp8KvCache(cache.codes[:, :, :, ::2], cache.scale)),
    ]
    for i, (what, call) in enumerate(bad):
        with pytest.raises(ValueError, match=what):
            call()
            pytest.fail(f"call {i} was not refused")


def test_attention_block_checks_its_weights(L):
    def weight(N, K):
        return binding.Fp8Weight(torch.zeros((N, K), dtype=torch.uint8), torch.ones(((N + 127) // 128, (K + 127) // 128)), N, K, pow2=True)

    rope = torch.zeros((10, 64))
    b = attention_fp8.AttentionFp8(weight(12 * 64, 256), weight(256, 8 * 64), 8, 2, rope)
    assert b.D == 64
    for Hq, H, out in ((8, 3, 512), (8, 2, 256), (7, 2, 448), (8, 0, 512)):
        with pytest.raises(ValueError):
            attention_fp8.AttentionFp8(weight(12 * 64, 256), weight(256, out), Hq, H, rope)


def test_rotary_table():
    t = binding.rotary_table(70000, 16, 500000.0, "cpu")
    for p, i in ((0, 0), (1, 3), (69999, 0), (69999, 7)):
        a = p * 500000.0 ** (-2 * i / 16)
        # an angle of 7e4 is known to 7e4 * 2^-53, the result rounded to FP32
        assert abs(float(t[p, i]) - math.cos(a)) <= 2.0 ** -24 + 1e-10 and abs(float(t[p, 8 + i]) - math.sin(a)) <= 2.0 ** -24 + 1e-10


def test_units_of_a_ragged_batch(tmp_path):
    """Every page that a batch touches belongs to a unit, and each unit finds its sequence (host build of the device code)."""
    src = tmp_path / "t.cpp"
    src.write_text('''
#include "kv_index.h"
extern "C" int sequence(long long u, int B, int size, int extra, const long long* cu) {
  return zq::kv::unit_sequence(u, B, size, extra, [&](int b) { return cu[b]; });
}
extern "C" long long base(long long row, long long b, int size, int extra) { return zq::kv::unit_base(row, b, size, extra); }
''')
    so = tmp_path / "t.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2307_09782_b200", "csrc"), str(src),
                    "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.base.restype = C.c_longlong
    lib.base.argtypes = [C.c_longlong, C.c_longlong, C.c_int, C.c_int]
    lib.sequence.argtypes = [C.c_longlong, C.c_int, C.c_int, C.c_int, C.c_void_p]
    g = torch.Generator().manual_seed(0)
    for size, extra, big in ((16, 2, 0), (64, 2, 0), (128, 1, 0), (32, 1, 0), (64, 2, (1 << 31) - 1000)):
        new = torch.randint(0, 150, (40,), generator=g).tolist()
        start = torch.randint(0, 300, (40,), generator=g).tolist()
        if big:
            new[3] = big - sum(new)  # offsets close to 2^31
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        arr = (C.c_longlong * 41)(*cu)
        total = lib.base(cu[-1], 40, size, extra)
        seen = 0
        for b in range(40):
            first = lib.base(cu[b], b, size, extra)
            off = start[b] % size if extra == 2 else 0
            pages = -(-(off + new[b]) // size) if new[b] else 0
            for i in ([0, pages // 2, pages - 1] if pages > 20 else range(pages)):
                assert 0 <= first + i < total
                assert lib.sequence(first + i, 40, size, extra, arr) == b
                seen += 1
        assert seen > 40


def test_plain_forms_agree_with_torch():
    """The 64-bit forms on the CPU against torch's own softmax and a table lookup of E4M3."""
    codes, scale, table, lens, cu = R.batch([37, 5], [3, 5], 2, 64, 16, dev="cpu")
    q = R.heads(8, 4, 64, 7, dev="cpu")
    o, lse, _ = R.attention(codes, scale, q, table, lens, cu, 0.125, True, 0)
    kv = R.gather(codes, scale, table[0].tolist(), 37)
    for i in range(3):
        for h in range(4):
            s = (kv[0, h // 2][:35 + i] @ q[i, h].double()) * 0.125
            assert torch.allclose(o[i, h], torch.softmax(s, 0) @ kv[1, h // 2][:35 + i], rtol=1e-12)
            assert torch.allclose(lse[i, h], torch.logsumexp(s, 0), rtol=1e-12)
    x = torch.randn(3, 64) * 100
    c = R.codes_of(x, torch.tensor(1.0))
    grid = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    grid = grid[torch.isfinite(grid)]
    assert torch.equal((x.clamp(-448, 448)[..., None] - grid).abs().min(-1).values, (x.clamp(-448, 448) - c.view(torch.float8_e4m3fn).float()).abs())
