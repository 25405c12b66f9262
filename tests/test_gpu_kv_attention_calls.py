"""The attention half of a decoder layer as programs call it: the block with its cache over prompts and decoding steps, streams,
graphs, threads, large caches, many sequences.  Tolerances as in test_gpu_kv_attention.py."""
import threading

import pytest
import torch

import kv_ref as R
from paper_2307_09782_b200 import binding
from paper_2307_09782_b200.attention_fp8 import AttentionFp8
from test_gpu_kv_attention import attn_tolerance

pytestmark = pytest.mark.gpu
K, HQ, H, D = 256, 8, 2, 64


def block(seed=0, **kw):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    return AttentionFp8.from_weights(normal((HQ + 2 * H) * D, K) * K ** -0.5, normal(K, HQ * D) * (HQ * D) ** -0.5, HQ, H,
                                     binding.rotary_table(4096, D), q_norm=1 + 0.1 * normal(D), k_norm=1 + 0.1 * normal(D), **kw)


def inputs(T, seed=1):
    return torch.randn((T, K), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


def strung(b, x, cache, pages, lens, positions, cu=None):
    """The block's calls one by one, into tensors of their own."""
    T = x.shape[0]
    qkv = binding.fp8_block_linear(b.qkv, x=x, mode=b.mode, out_dtype=torch.bfloat16).view(T, HQ + 2 * H, D)
    q, k = binding.qk_norm_rope(qkv[:, :HQ], qkv[:, HQ:HQ + H], b.table, positions, wq=b.q_norm, wk=b.k_norm)
    binding.kv_cache_write(cache, k, qkv[:, HQ + H:].contiguous(), pages, lens, cu=cu, mode=b.cache_mode)
    o = binding.kv_attention(cache, q, pages, lens, cu=cu, window=b.window)
    return binding.fp8_block_linear(b.out, x=o.flatten(1), mode=b.mode, out_dtype=torch.bfloat16), q, o


@pytest.mark.parametrize("mode,cache_mode,window", [("none", "none", 0), ("M1", "M1", 30)])
def test_block_over_prompts_and_decoding(mode, cache_mode, window):
    """Three users: prompts of 100, 3 and 40 tokens at once, then steps of one token each.  The block gives what its calls give one
    by one, and the attention is that of 64 bits over what the cache holds."""
    b = block(mode=mode, cache_mode=cache_mode, window=window)
    caches = [b.new_cache(40, 16), b.new_cache(40, 16)]
    order = torch.randperm(40, generator=torch.Generator().manual_seed(3))[:30].to(torch.int32).view(3, 10)
    pages = order.cuda()
    new = [100, 3, 40]
    lens = list(new)
    for step in range(12):
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        positions = torch.cat([torch.arange(L - n, L) for L, n in zip(lens, new)]).to(torch.int32).cuda()
        x = inputs(cu[-1], step)
        args = (pages, R.ints(lens), positions)
        cu_ = R.ints(cu) if step == 0 else None
        y = b.forward(x, caches[0], *args, cu=cu_)
        ref, q, o = strung(b, x, caches[1], *args, cu=cu_)
        assert torch.equal(y, ref) and torch.equal(caches[0].codes, caches[1].codes) and torch.equal(caches[0].scale, caches[1].scale)
        o64, _, bound = R.attention(caches[0].codes, caches[0].scale, q, pages, lens, cu, D ** -0.5, True, window)
        assert ((o.to(R.F64) - o64).abs() <= attn_tolerance(o64, bound, torch.bfloat16)).all()
        new = [1, 1, 1]
        lens = [L + 1 for L in lens]


def test_prompt_in_chunks():
    """A prompt in chunks that end at pages leaves the cache of the whole prompt, and the same attention."""
    b = block()
    whole, parts = b.new_cache(20, 32), b.new_cache(20, 32)
    pages = torch.arange(20, dtype=torch.int32, device="cuda").view(1, 20)
    x, positions = inputs(600), torch.arange(600, dtype=torch.int32, device="cuda")
    y = b.forward(x, whole, pages, R.ints([600]), positions, cu=R.ints([0, 600]))
    got = [b.forward(x[i:j], parts, pages, R.ints([j]), positions[i:j], cu=R.ints([0, j - i])) for i, j in ((0, 64), (64, 544), (544, 600))]
    assert torch.equal(whole.codes, parts.codes) and torch.equal(whole.scale, parts.scale)
    # o is rounded to bf16 (half a step more or less on either side), then to E4M3 by the projection: 2^-4 of a product at most
    assert ((torch.cat(got) - y).float().norm() <= 2.0 ** -4 * y.float().norm())


def test_captured_steps():
    """Decoding steps replayed from a graph, with lengths and positions written between replays, and eager calls among them."""
    b = block()
    eager, graphed = b.new_cache(12, 16), b.new_cache(12, 16)
    pages = torch.arange(12, dtype=torch.int32, device="cuda").view(2, 6)
    lens, positions, x = R.ints([1, 1]), R.ints([0, 0]), inputs(2)
    b.forward(x, graphed, pages, lens, positions)  # (attributes are set, weights looked at)
    graphed.codes.zero_()
    graphed.scale.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = b.forward(x, graphed, pages, lens, positions)
    for step in range(1, 40):
        lens.fill_(step)
        positions.fill_(step - 1)
        x.copy_(inputs(2, step))
        ref = b.forward(x, eager, pages, lens, positions)
        g.replay()
        assert torch.equal(y, ref), step
    assert torch.equal(eager.codes, graphed.codes) and torch.equal(eager.scale, graphed.scale)


def test_two_graphs_do_not_share():
    """Two captured calls of other sizes, replayed in turn and at once on two streams."""
    cases = [([900, 33], [1, 1]), ([700], [300])]
    todo = []
    for i, (lens, new) in enumerate(cases):
        codes, scale, table, lens, cu = R.batch(lens, new, H, D, 32, seed=i)
        q = R.heads(cu[-1], HQ, D, 5 + i)
        args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
        cu_ = R.ints(cu)
        ref = binding.kv_attention(*args, cu=cu_)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = binding.kv_attention(*args, cu=cu_)
        todo.append((g, out, ref, args, cu_))  # (a graph keeps its own memory, not its inputs)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for (g, out, *_), s in zip(todo, streams):
            with torch.cuda.stream(s):
                out.zero_()
                g.replay()
    torch.cuda.synchronize()
    for _, out, ref, *_ in todo:
        assert torch.equal(out, ref)


def test_backward_captured_beside_eager():
    q, k = R.heads(50, HQ, D, 1), R.heads(50, H, D, 2)
    dq, dk = R.heads(50, HQ, D, 3), R.heads(50, H, D, 4)
    w = torch.ones(D, device="cuda")
    table, positions = binding.rotary_table(64, D), torch.arange(50, dtype=torch.int32, device="cuda")
    args = (dq, dk, q, k, table, positions)
    first = binding.qk_norm_rope_backward(*args, wq=w, wk=w)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = binding.qk_norm_rope_backward(*args, wq=w, wk=w)
    again = binding.qk_norm_rope_backward(*args, wq=w, wk=w)
    g.replay()
    for a, b_, c in zip(first, again, got):
        assert torch.equal(a, b_) and torch.equal(a, c)


def test_other_stream_and_threads():
    """Calls without a workspace on streams of their own and, from several threads, on one stream."""
    jobs = []
    for i in range(4):
        codes, scale, table, lens, cu = R.batch([500 + 100 * i, 40], [1 + 30 * i, 2], H, D, 16, seed=i)
        q = R.heads(cu[-1], HQ, D, i)
        args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
        jobs.append((args, R.ints(cu), binding.kv_attention(*args, cu=R.ints(cu))))
    torch.cuda.synchronize()
    wrong = []

    def run(job, stream):
        args, cu, ref = job
        with torch.cuda.stream(stream):
            for _ in range(20):
                if not torch.equal(binding.kv_attention(*args, cu=cu), ref):
                    wrong.append(1)
    shared = torch.cuda.Stream()
    for streams in ([torch.cuda.Stream() for _ in jobs], [shared] * len(jobs)):
        ts = [threading.Thread(target=run, args=(j, s)) for j, s in zip(jobs, streams)]
        [t.start() for t in ts]
        [t.join() for t in ts]
    assert not wrong


@pytest.mark.parametrize("n", [1, 3, 200])
def test_cache_beyond_32_bits(n):
    """Pages 2^32 bytes and more into the cache."""
    page, pages = 128, 18000
    cache = binding.Fp8KvCache(torch.zeros((pages, 2, 8, page, 128), dtype=torch.uint8, device="cuda"),
                               torch.zeros((pages, 2, 8), device="cuda"))
    assert cache.codes.numel() > 2 ** 32
    L = 300
    table = R.ints([[pages - 1, 3, pages - 2]])
    k, v = R.heads(L, 8, 128, 1), R.heads(L, 8, 128, 2)
    cu = R.ints([0, L])
    binding.kv_cache_write(cache, k, v, table, R.ints([L]), cu=cu)
    small = torch.zeros((3, 2, 8, page, 128), dtype=torch.uint8, device="cuda"), torch.zeros((3, 2, 8), device="cuda")
    expect = R.write(*small, k, v, R.ints([[0, 1, 2]]), [L], [0, L], "none")
    where = [pages - 1, 3, pages - 2]
    assert torch.equal(cache.codes[where], expect[0]) and torch.equal(cache.scale[where], expect[1])
    assert int(cache.codes.count_nonzero()) == int(expect[0].count_nonzero())
    q = R.heads(n, 16, 128, 3)
    got = binding.kv_attention(cache, q, table, R.ints([L]), cu=R.ints([0, n]))
    ref, _, bound = R.attention(*expect, q, R.ints([[0, 1, 2]]), [L], [0, n], 128 ** -0.5, True, 0)
    assert ((got.to(R.F64) - ref).abs() <= attn_tolerance(ref, bound, torch.bfloat16)).all()
    kk, vv = binding.kv_cache_read(cache, table, cu, L)
    small = binding.kv_cache_read(binding.Fp8KvCache(*expect), R.ints([[0, 1, 2]]), cu, L)
    assert torch.equal(kk, small[0]) and torch.equal(vv, small[1])


def test_many_sequences():
    """More sequences than a block has threads, most of them short, some empty, a few with many rows."""
    g = torch.Generator().manual_seed(0)
    lens = torch.randint(0, 40, (1500,), generator=g).tolist()
    new = [min(L, 1 if i % 3 else 2) for i, L in enumerate(lens)]
    lens[700], new[700] = 300, 90
    lens[1499], new[1499] = 200, 33
    codes, scale, table, lens, cu = R.batch(lens, new, 1, 64, 16)
    q = R.heads(cu[-1], 2, 64, 7)
    got, lse = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), lse=True)
    ref, ref_lse, bound = R.attention(codes, scale, q, table, lens, cu, 0.125, True, 0)
    assert ((got.to(R.F64) - ref).abs() <= attn_tolerance(ref, bound, torch.bfloat16)).all()
    assert torch.allclose(lse.to(R.F64), ref_lse, rtol=0, atol=1e-3)
    k, v = R.heads(cu[-1], 1, 64, 8), R.heads(cu[-1], 1, 64, 9)
    expect = R.write(codes, scale, k, v, table, lens, cu, "none")
    binding.kv_cache_write(binding.Fp8KvCache(codes, scale), k, v, table, R.ints(lens), cu=R.ints(cu))
    assert torch.equal(codes, expect[0]) and torch.equal(scale.nan_to_num(nan=-1), expect[1].nan_to_num(nan=-1))


@pytest.mark.parametrize("G,n", [(1, 64), (1, 65), (64, 1), (65, 1), (16, 4), (13, 5), (5, 13), (1, 128), (1, 129), (1, 256), (1, 257), (3, 86)])
def test_rows_at_the_kernels_borders(G, n):
    codes, scale, table, lens, cu = R.batch([700, 129], [n, 1], 2, 128, 64)
    q = R.heads(cu[-1], 2 * G, 128, 7)
    got = binding.kv_attention(binding.Fp8KvCache(codes, scale), q, table, R.ints(lens), cu=R.ints(cu), out_dtype=torch.float32)
    ref, _, bound = R.attention(codes, scale, q, table, lens, cu, 128 ** -0.5, True, 0)
    assert ((got.to(R.F64) - ref).abs() <= attn_tolerance(ref, bound, torch.float32)).all()


def test_strides_and_workspace():
    """Queries that are part of wider rows, results into wider rows, one workspace for larger and smaller calls."""
    ws = binding.make_workspace(binding.kv_attention_workspace_bytes(400, 4, HQ, H, D))
    for lens, new in (([500], [400]), ([90, 700, 5], [1, 1, 1]), ([40, 300], [40, 3])):
        codes, scale, table, lens, cu = R.batch(lens, new, H, D, 32)
        T = cu[-1]
        q = R.heads(T, HQ, D, 7, 6)
        wide = torch.full((T, HQ + 3, D), 7.0, dtype=torch.bfloat16, device="cuda")
        args = (binding.Fp8KvCache(codes, scale), q, table, R.ints(lens))
        binding.kv_attention(*args, cu=R.ints(cu), out=wide[:, 2:2 + HQ], workspace=ws)
        assert torch.equal(wide[:, 2:2 + HQ], binding.kv_attention(*args[:1], q.contiguous(), *args[2:], cu=R.ints(cu)))
        assert (wide[:, :2] == 7).all() and (wide[:, 2 + HQ:] == 7).all()
        assert binding.device_status(ws)[0] == 0


def test_tensors_elsewhere_are_refused():
    codes, scale, table, lens, cu = R.batch([40], [1], H, D, 16)
    q = R.heads(1, HQ, D, 7)
    cache = binding.Fp8KvCache(codes, scale)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.kv_attention(cache, q, table.cpu(), R.ints(lens))
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding.kv_attention(cache, q, table, R.ints(lens), workspace=torch.zeros(1 << 26, dtype=torch.uint8))
    with pytest.raises(binding.ZqError):
        binding.kv_attention(cache, q, table, R.ints(lens), workspace=torch.zeros(1 << 12, dtype=torch.uint8, device="cuda"))
