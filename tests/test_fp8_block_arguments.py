"""Arguments that the binding of the FP8 operators must refuse, or look after, before anything is launched (no GPU needed)."""
import copy
import pickle
import threading

import pytest
import torch

import __graft_entry__ as entry
from paper_2307_09782_b200 import binding, gated_ffn

u8, f32, bf = torch.uint8, torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def L():
    entry.build()
    return binding.lib()


def weight(N, K, parts=1, **kw):
    lead = (parts,) if parts > 1 else ()
    nb, kb = (N + 127) // 128, (K + 127) // 128
    return binding.Fp8Weight(torch.zeros((*lead, N, K), dtype=u8), torch.ones((*lead, nb, kb)), N, K, parts, **kw)


# ---- result types ----------------------------------------------------------------------------------------------------
OTHER_TYPES = [torch.float16, torch.float64, torch.uint8, torch.float8_e4m3fn, torch.int32]


@pytest.mark.parametrize("dtype", OTHER_TYPES)
def test_result_types(dtype):
    """The library writes FP32 or bf16: into a tensor of another type it would write wrong bits, or beyond its end."""
    x = torch.zeros((4, 64), dtype=bf)
    work = torch.zeros(256, dtype=u8)
    gu, down = weight(32, 64, 2), weight(64, 32)
    gut, dnt = weight(64, 32, 2), weight(32, 64)
    saved = torch.zeros(binding.fp8_gated_ffn_saved_bytes(4, 64, 32), dtype=u8)
    ffn = gated_ffn.GatedFfnFp8(gu, down)
    ffn.gate_up_t, ffn.down_t = gut, dnt
    ffn.workspace = lambda M: work
    calls = [lambda: binding.fp8_block_linear(weight(32, 64), x=x, out_dtype=dtype, workspace=work),
             lambda: binding.fp8_block_linear(weight(32, 64), x=x, y=torch.zeros((4, 32)).to(dtype), workspace=work),
             lambda: binding.fp8_weight_grad(torch.zeros((4, 8), dtype=bf), binding.Fp8Block(torch.zeros((4, 64), dtype=u8),
                                                                                             torch.ones((1, 4))),
                                             out_dtype=dtype, workspace=work),
             lambda: binding.fp8_gated_ffn(gu, down, x, out_dtype=dtype, workspace=work),
             lambda: binding.fp8_gated_ffn_backward(gut, dnt, x, saved, out_dtype=dtype, workspace=work),
             lambda: ffn.forward(x, out_dtype=dtype), lambda: ffn.forward_train(x, out_dtype=dtype),
             lambda: ffn.backward(x, saved, out_dtype=dtype)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="out_dtype"):
            call()
            pytest.fail(str(i))


@pytest.mark.parametrize("dtype", OTHER_TYPES)
def test_result_types_w4a8(dtype):
    w = binding.PackedWeight(torch.zeros(8704, dtype=u8), torch.zeros((128, 1), dtype=u8), torch.ones(128), 128, 128, 128,
                             binding.SCALE_M2)
    q, sx, work = torch.zeros((4, 128), dtype=u8), torch.ones(4), torch.zeros(256, dtype=u8)
    y = torch.zeros((4, 128)).to(dtype)
    for call in (lambda **kw: binding.w4a8_linear(w, q=q, sx=sx, workspace=work, **kw),
                 lambda **kw: binding.w4a8_linear_noalloc(w, q=q, sx=sx, **kw)):
        for kw in (dict(out_dtype=dtype), dict(y=y)):
            with pytest.raises(ValueError, match="out_dtype"):
                call(**kw)


# ---- workspaces that are kept ------------------------------------------------------------------------------------------
@pytest.fixture
def kept(monkeypatch):
    """The workspaces that the binding keeps, on the CPU, from an empty start."""
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_capturing", lambda: False, raising=False)
    monkeypatch.setattr(binding, "make_workspace", lambda n, device=None: torch.zeros(n, dtype=u8))
    monkeypatch.setattr(binding, "_fp8_workspaces", type(binding._fp8_workspaces)())
    return torch.device("cpu")


SEQUENCES = [[(2048, 512), (300, 4096)], [(100, 1024), (27, 4096)], [(8192, 7168), (2075, 28672)], [(8192, 256), (700, 4096)],
             [(1000, 16), (1, 100_000)], [(0, 16), (1, 16), (3, 128), (2, 4096), (1, 8192), (64, 16)]]


@pytest.mark.parametrize("calls", SEQUENCES)
def test_kept_workspace_is_large_enough(kept, L, calls):
    for M, K in calls:
        ws = binding._fp8_workspace(None, M, K, kept)
        assert ws.numel() >= L.zq_fp8_block_workspace_bytes(M, K), (M, K)


def test_workspace_need(L):
    for M in (0, 1, 2, 7, 64, 333, 4096, 100_003):
        for K in (16, 128, 144, 4096, 11008, 28672):
            assert binding._fp8_workspace_need(M, K) == L.zq_fp8_block_workspace_bytes(M, K)


def test_captured_calls_keep_nothing(kept, monkeypatch):
    """A captured call's workspace is neither the kept one, which may be given back while the graph lives, nor kept."""
    monkeypatch.setattr(binding, "_capturing", lambda: False)
    ffn = gated_ffn.GatedFfnFp8(weight(32, 64, 2), weight(64, 32))
    eager = binding._fp8_workspace(None, 8, 64, kept), ffn.workspace(8)
    monkeypatch.setattr(binding, "_capturing", lambda: True)
    captured = [binding._fp8_workspace(None, 8, 64, kept), ffn.workspace(8), binding._fp8_workspace(None, 8, 64, kept),
                ffn.workspace(8)]
    assert len({t.data_ptr() for t in (*eager, *captured)}) == 6
    monkeypatch.setattr(binding, "_capturing", lambda: False)
    assert binding._fp8_workspace(None, 8, 64, kept) is eager[0] and ffn.workspace(8) is eager[1]


def test_threads_share_no_workspace(kept):
    """Threads can share a stream (all start on the default one) and their calls' kernels mix there."""
    ffn = gated_ffn.GatedFfnFp8(weight(32, 64, 2), weight(64, 32))

    def both():
        return binding._fp8_workspace(None, 8, 64, kept), ffn.workspace(8)

    mine, others = both(), []
    t = threading.Thread(target=lambda: others.extend([*both(), *both()]))
    t.start()
    t.join()
    assert others[0] is others[2] and others[1] is others[3]
    assert len({b.data_ptr() for b in (*mine, *others)}) == 4
    assert both()[0] is mine[0] and both()[1] is mine[1]


def test_block_can_be_copied(kept):
    ffn = gated_ffn.GatedFfnFp8(weight(32, 64, 2), weight(64, 32))
    ws = ffn.workspace(8)
    for other in (copy.deepcopy(ffn), pickle.loads(pickle.dumps(ffn))):
        assert torch.equal(other.down.codes, ffn.down.codes) and other.workspace(8).data_ptr() != ws.data_ptr()


# ---- scales that change ------------------------------------------------------------------------------------------------
def test_promise_ends_with_a_write(monkeypatch):
    """What is known of scales holds until they are written to, or others take their place."""
    monkeypatch.setattr(binding, "_capturing", lambda: False, raising=False)
    P2 = binding.SCALES_POW2
    writes = [lambda t: t.mul_(1.5), lambda t: t.copy_(torch.full_like(t, 3.0)), lambda t: t[0].fill_(0.7), lambda t: t.view(-1).add_(1)]
    for write in writes:
        w, q = weight(128, 128, pow2=True), binding.Fp8Block(torch.zeros((4, 128), dtype=u8), torch.ones((1, 4)), True)
        down = weight(128, 128, pow2=True)
        assert binding._scales("M1", w, None) == binding.SCALE_M1 | P2 and binding._scales("none", w, q) == P2
        write(q.scale)
        assert not q.pow2 and binding._scales("none", w, q) == 0
        q.pow2 = True  # told anew
        assert binding._scales("none", w, q) == P2
        write(w.scale)
        assert not w.pow2 and binding._scales("M1", w, None) == binding.SCALE_M1 and binding._scales("none", w, q) == 0
        assert binding._ffn_scales("M1", down, w) == binding.SCALE_M1 and binding._ffn_scales("M1", w, down) == binding.SCALE_M1
        w.scale = torch.ones((1, 1))
        w.pow2 = True
        assert binding._ffn_scales("M1", down, w) == binding.SCALE_M1 | P2
        w.scale = torch.full((1, 1), 1.5)
        assert not w.pow2
        q.scale = torch.full((1, 4), 1.5)
        assert not q.pow2


def test_promise_in_inference_mode():
    with torch.inference_mode():
        w = weight(128, 128, pow2=True)
        assert binding._scales("M1", w, None) == binding.SCALE_M1 | binding.SCALES_POW2
    assert w.pow2 is True


# ---- sizes ---------------------------------------------------------------------------------------------------------------
@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: only a machine without a GPU stops in time")
def test_no_tokens_are_not_refused(L):
    """The block's backward pass, and the weight gradient of several parts, of a batch without tokens: whatever stops them here, it
    is not the sizes."""
    P, K, F, N = 0x10000, 64, 32, 48
    ws = binding.fp8_gated_ffn_workspace_bytes(0, K, F, N, True)
    assert L.zq_fp8_gated_ffn_backward(None, N, 0, 0, K, F, N, None, None, None, None, None, 0, None, P, P, 1, P, ws, None) in (-6, -7)
    assert L.zq_fp8_weight_grad(None, F, 0, 2, None, None, 0, F, K, P, 1, P, ws, None) in (-6, -7)
    assert L.zq_fp8_weight_grad(P, F, 0, 2, P, P, 1, F, K, P, 1, P, ws, None) == -2  # with tokens: all parts in one place


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: only a machine without a GPU stops in time")
def test_one_matrix_has_no_stride(L):
    """Of one gradient matrix nothing is refused for where a second one would be."""
    P, ws = 0x10000, binding.fp8_block_linear_workspace_bytes(0, 0, 16)
    for stride in (0, 20, 21, -8):
        assert L.zq_fp8_weight_grad(P, 24, stride, 1, P, P, 1, 20, 64, P, 0, P, ws, None) in (-6, -7)
    assert L.zq_fp8_weight_grad(P, 24, 20, 2, P, P, 1, 20, 64, P, 0, P, ws, None) == -3


# ---- the caller's workspace ----------------------------------------------------------------------------------------------
def test_callers_workspace(kept):
    """Bytes in one piece, in the GPU's memory: its length is taken for granted in the library."""
    for ws, what in ((torch.zeros(1 << 20, dtype=u8), "CUDA"), (torch.zeros(1 << 20), "workspace"),
                     (torch.zeros(1, dtype=u8).expand(1 << 20), "workspace"), (torch.zeros(1 << 20, dtype=u8)[::2], "workspace")):
        with pytest.raises(ValueError, match=what):
            binding._fp8_workspace(ws, 4, 64, kept)


class On:
    """A tensor as far as its place goes."""

    def __init__(self, d):
        self.device, self.shape, self.is_cuda, self.get_device = torch.device("cuda", d), (2, 3), True, lambda: d


def test_other_devices_are_refused(monkeypatch):
    """Kernels run on the current device and its stream: all tensors have to be there."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    binding._on_gpu(On(1), On(1))
    for tensors in ((On(0), On(0)), (On(1), On(0)), (On(0), On(1)), (On(1), On(1), On(2))):
        with pytest.raises(ValueError, match="current device is cuda:1"):
            binding._on_gpu(*tensors)
    with pytest.raises(ValueError, match="CUDA tensor"):
        binding._on_gpu(On(1), torch.zeros(1))


@pytest.mark.parametrize("writes", [0, 1, 2, 3])
def test_promise_of_copies(writes):
    """A copy starts with what is known of the original, and its own writes end it, however many the original had seen."""
    for make in (lambda: weight(128, 128), lambda: binding.Fp8Block(torch.zeros((4, 128), dtype=u8), torch.ones((1, 4)))):
        for dup in (copy.deepcopy, lambda v: pickle.loads(pickle.dumps(v)), copy.copy):
            w = make()
            for _ in range(writes):
                w.scale.mul_(2.0)
            w.pow2 = True
            other = dup(w)
            assert other.pow2 is True and torch.equal(other.scale, w.scale)
            for _ in range(4):
                other.scale.mul_(1.5)
                assert other.pow2 is False
            assert w.pow2 is (dup is not copy.copy)
            w.scale.mul_(1.5)
            assert w.pow2 is False and dup(w).pow2 is False
