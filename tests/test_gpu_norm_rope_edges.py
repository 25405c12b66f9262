"""Norms with the position rotation where a warp works on several units, where heads do not fill a unit, and on numbers that have to come
out as they went in.  Tolerances as in test_gpu_kv_attention.py."""
import pytest
import torch

import kv_ref as R
from paper_2307_09782_b200 import binding
from test_gpu_kv_attention import half_step, norm_inputs

pytestmark = pytest.mark.gpu
EPS = 1e-6


def check_forward(case, eps=EPS):
    q, k, wq, wk, table, positions = norm_inputs(case)
    yq, yk = binding.qk_norm_rope(q, k, table, positions, wq=wq, wk=wk, eps=eps, pairs=case[5])
    for x, w, y in ((q, wq, yq), (k, wk, yk)):
        ref = R.norm_rope(x.to(R.F64), None if w is None else w.to(R.F64), table, positions, eps, case[5])
        big = ref.abs().amax(-1, keepdim=True)
        assert ((y.to(R.F64) - ref).abs() <= half_step(torch.bfloat16) * ref.abs() + 2.0 ** -20 * big).all()


def check_backward(case, eps=EPS):
    q, k, wq, wk, table, positions = norm_inputs(case)
    T, Hq, H, D = case[:4]
    dq, dk = R.heads(T, Hq, D, 11, 2), R.heads(T, H, D, 12)
    got = binding.qk_norm_rope_backward(dq, dk, q, k, table, positions, wq=wq, wk=wk, eps=eps, pairs=case[5])
    for x, w, dy, dx, dw in ((q, wq, dq, got[0], got[2]), (k, wk, dk, got[1], got[3])):
        x64 = x.to(R.F64).requires_grad_()
        w64 = None if w is None else w.to(R.F64).requires_grad_()
        R.norm_rope(x64, w64, table, positions, eps, case[5]).backward(dy.to(R.F64))
        rms = (x.to(R.F64).square().mean(-1, keepdim=True) + eps).sqrt()
        length = dy.to(R.F64).norm(dim=-1, keepdim=True)
        size = dy.to(R.F64).abs().amax(-1, keepdim=True) if w is None else length * 2 * w.abs().max() / rms
        assert ((dx.to(R.F64) - x64.grad).abs() <= half_step(torch.bfloat16) * x64.grad.abs() + 2.0 ** -19 * size).all()
        if w is None:
            assert dw is None
        else:
            terms = (length * (x.to(R.F64) / rms).abs()).sum((0, 1))
            assert ((dw.to(R.F64) - w64.grad).abs() <= 2.0 ** -20 * terms).all()


@pytest.mark.parametrize("Hq,H,D", [(1, 1, 128), (2, 1, 64), (12, 12, 64), (9, 3, 128), (16, 8, 128)])
def test_no_epsilon(Hq, H, D):
    """eps = 0, which only a head of zeros cannot take; heads that fill a unit and heads that do not."""
    case = (37, Hq, H, D, D, "halves", True, 1)
    check_forward(case, 0.0)
    check_backward(case, 0.0)


def test_features_that_are_not_rotated_pass_unchanged():
    """Every bf16 number there is, zeros of both signs among them, in both directions and both pairings; NaN as some NaN."""
    T, D, rot = 1366, 64, 16
    x = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda")
    bits = torch.arange(T * (D - rot), device="cuda").to(torch.int16).view(T, 1, D - rot)
    x.view(torch.int16)[..., rot:] = bits
    nan = x[..., rot:].isnan()
    table = binding.rotary_table(100, rot)
    positions = torch.arange(T, device="cuda", dtype=torch.int32) % 100
    for pairs in ("halves", "neighbours"):
        for y in (*binding.qk_norm_rope(x, x, table, positions, pairs=pairs),
                  *binding.qk_norm_rope_backward(x, x, x, x, table, positions, pairs=pairs)[:2]):
            assert torch.equal(y.view(torch.int16)[..., rot:][~nan], bits[~nan]) and y[..., rot:][nan].isnan().all()
            assert not y[..., :rot].any()



WALKS = [
    # more units than the device has warps, several units per token and kind
    (2500, 20, 3, 128, 128, "halves", True, 2),
    (2500, 20, 3, 128, 32, "neighbours", True, 0),
    (2501, 20, 3, 64, 48, "halves", True, 1),
    (3001, 17, 33, 64, 64, "neighbours", False, 0),
]


@pytest.mark.parametrize("case", WALKS)
def test_several_units_per_warp(case):
    check_forward(case)
    check_backward(case)


@pytest.mark.parametrize("case", [WALKS[0], WALKS[3]])
def test_several_units_per_warp_in_place_and_on_parts(case):
    """In place as out of place; and what is computed for a part of the tokens does not depend on the others."""
    q, k, wq, wk, table, positions = norm_inputs(case)
    kw = dict(wq=wq, wk=wk, pairs=case[5])
    whole = binding.qk_norm_rope(q, k, table, positions, **kw)
    part = binding.qk_norm_rope(q[77:131], k[77:131], table, positions[77:131].contiguous(), **kw)
    assert all(torch.equal(w[77:131], p) for w, p in zip(whole, part))
    binding.qk_norm_rope(q, k, table, positions, **kw, out=(q, k))
    assert torch.equal(q, whole[0]) and torch.equal(k, whole[1])
