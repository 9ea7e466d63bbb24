"""Gradient norm over a list of tensors and clipping by it, against the float64 oracle."""

import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo
from paper_2605_17862_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def _ws():
    n = fb.fopd_grad_workspace_bytes()
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device=DEV)
    off = (-ws.data_ptr()) % 256
    ws = ws[off:off + n]
    fb.fopd_workspace_init(ws)
    return ws


def _scalars():
    return torch.full((1,), 99.0, dtype=torch.float64, device=DEV), torch.full((1,), 99.0, device=DEV), torch.full((1,), 99.0, device=DEV)


def _tensors(shapes, dtypes, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * scale * (1 + i % 3)).to(dt).to(DEV) for i, (s, dt) in enumerate(zip(shapes, dtypes))]


def _f64(t):
    return t.double().cpu().numpy()


def _check(grads, outs, before, max_norm, sum_sq, norm, coef):
    # (the entry point's two numbers are floats: what it was given is their rounding, up to 2^-24 away)
    total, n, c, want = oo.grad_clip(before, float(np.float32(max_norm)), float(np.float32(EPS)))
    count = sum(b.size for b in before)
    assert abs(float(sum_sq) - total) <= count * 2.0 ** -52 * total          # 64-bit squares and additions
    assert abs(float(norm) - n) <= 2.0 ** -24 * 1.01 * n
    assert abs(float(coef) - c) <= 2.0 ** -24 * 1.01 * c
    for o, w in zip(outs, want):
        # the coefficient's rounding, the product's in 32 bits, the result's
        tol = np.abs(w) * (2.0 ** -23 * 1.01 + (2.0 ** -8 * 1.01 if o.dtype is torch.bfloat16 else 0.0))
        tol += 2.0 ** -149 if o.dtype is torch.float32 else 2.0 ** -133
        assert (np.abs(_f64(o) - w) <= tol).all()


# (no tensor at all, one table, its last entry, more tables than one, more than one table with empty tensors between)
SHAPES = [[(1,)], [(7,), (8,), (0,), (9, 0), (3, 5)], [(8191,), (8192,), (8193,)], [(300, 500), (16385,), (2, 3, 70)],
          [(1000, 1000)] + 60 * [(33,)], 130 * [(257,)], 48 * [(3,)], 49 * [(3,), (0,)]]


@pytest.mark.parametrize("shapes", SHAPES)
@pytest.mark.parametrize("kinds", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("place", ["in_place", "out", "cast"])
def test_norm_and_clip_against_the_oracle(shapes, kinds, place):
    pick = {"f32": [torch.float32], "bf16": [torch.bfloat16], "mixed": [torch.float32, torch.bfloat16]}[kinds]
    grads = _tensors(shapes, [pick[i % len(pick)] for i in range(len(shapes))], seed=len(shapes))
    before = [_f64(g) for g in grads]
    other = {torch.float32: torch.bfloat16, torch.bfloat16: torch.float32}
    outs = {"in_place": None, "out": [torch.empty_like(g) for g in grads],
            "cast": [torch.empty_like(g, dtype=other[g.dtype]) for g in grads]}[place]
    tensors = fb.grad_tensors(grads, outs)
    sum_sq, norm, coef = _scalars()
    n = math.sqrt(sum((b ** 2).sum() for b in before))
    for most in (4.0 * n, 0.3 * n):                                          # not clipped, then clipped
        fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
        fb.fopd_grad_clip(tensors, sum_sq, most, EPS, coef)
        _check(grads, grads if outs is None else outs, before, most, sum_sq, norm, coef)
        if most > n:
            assert float(coef) == 1.0
            for g, b in zip(grads, before):
                assert np.array_equal(_f64(g), b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("skip_in,skip_out", [(0, 0), (1, 0), (3, 3), (0, 5), (7, 2)])
def test_any_alignment_and_gaps_between_rows(dtype, skip_in, skip_out):
    g = torch.Generator().manual_seed(skip_in)
    flat = torch.randn(40000, generator=g).to(dtype).to(DEV)
    out = torch.full((40000,), 7.0, dtype=dtype, device=DEV)
    grads = [flat[skip_in:skip_in + 20011]]
    outs = [out[skip_out:skip_out + 20011]]
    wide = torch.randn(37, 301, generator=g).to(dtype).to(DEV)
    wide_out = torch.full((37, 310), 7.0, dtype=dtype, device=DEV)
    grads.append(wide[:, 1:290])                                             # 289 of 301 columns
    outs.append(wide_out[:, skip_out:skip_out + 289])
    whole = torch.randn(37, 64, generator=g).to(dtype).to(DEV)               # without gaps on one side only
    grads.append(whole)
    outs.append(torch.full((37, 72), 7.0, dtype=dtype, device=DEV)[:, :64])
    before = [_f64(t) for t in grads]
    tensors = fb.grad_tensors(grads, outs)
    sum_sq, norm, coef = _scalars()
    fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
    fb.fopd_grad_clip(tensors, sum_sq, 5.0, EPS, coef)
    _check(grads, outs, before, 5.0, sum_sq, norm, coef)
    assert bool((out[:skip_out] == 7.0).all()) and bool((out[skip_out + 20011:] == 7.0).all())
    assert bool((wide_out[:, :skip_out] == 7.0).all()) and bool((wide_out[:, skip_out + 289:] == 7.0).all())
    # in place: the gaps stay
    edge = wide[:, 290:].clone()
    fb.fopd_grad_clip(fb.grad_tensors(grads), sum_sq, 5.0, EPS, coef)
    _check(grads, grads, before, 5.0, sum_sq, norm, coef)
    assert torch.equal(wide[:, 290:], edge)


def test_squares_neither_vanish_nor_overflow():
    grads = [torch.full((1000,), 1e-30, device=DEV), torch.full((10,), 3e30, device=DEV)]
    sum_sq, norm, coef = _scalars()
    fb.fopd_grad_norm(fb.grad_tensors(grads[:1]), sum_sq, norm, _ws())
    assert float(norm) == pytest.approx(1e-30 * math.sqrt(1000), rel=1e-6)
    fb.fopd_grad_norm(fb.grad_tensors(grads[1:]), sum_sq, norm, _ws())
    assert float(norm) == pytest.approx(3e30 * math.sqrt(10), rel=1e-6)
    fb.fopd_grad_clip(fb.grad_tensors(grads[1:]), sum_sq, 1.0, 0.0, coef)
    assert torch.allclose(grads[1], torch.full((10,), 1 / math.sqrt(10), device=DEV), rtol=1e-6)


def test_no_tensors_empty_tensors_and_zero_gradients():
    for grads in ([], [torch.empty(0, device=DEV)], [torch.zeros(5, device=DEV)]):
        sum_sq, norm, coef = _scalars()
        tensors = fb.grad_tensors(grads)
        fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
        fb.fopd_grad_clip(tensors, sum_sq, 1.0, EPS, coef)
        assert (float(sum_sq), float(norm), float(coef)) == (0.0, 0.0, 1.0)


def test_nan_and_infinite_norms():
    for bad, c in ((float("nan"), float("nan")), (float("inf"), 0.0)):
        g = torch.ones(10000, device=DEV)
        g[8200] = bad
        h = torch.ones(5, dtype=torch.bfloat16, device=DEV)
        sum_sq, norm, coef = _scalars()
        tensors = fb.grad_tensors([g, h])
        fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
        fb.fopd_grad_clip(tensors, sum_sq, 1.0, EPS, coef)
        assert np.array_equal([float(coef)], [c], equal_nan=True)
        assert bool(torch.isnan(h).all()) if math.isnan(c) else bool((h == 0).all())
        assert math.isnan(float(g[8200])) and (math.isnan(float(g[0])) if math.isnan(c) else float(g[0]) == 0.0)


def test_lists_in_parts_add_up():
    grads = _tensors([(3000,), (40, 50), (123,)], 3 * [torch.float32], seed=3)
    sum_sq, norm, _ = _scalars()
    ws = _ws()
    fb.fopd_grad_norm(fb.grad_tensors(grads), sum_sq, norm, ws)
    parts, norm_parts, _ = _scalars()
    fb.fopd_grad_norm(fb.grad_tensors(grads[:1]), parts, None, ws)
    fb.fopd_grad_norm(fb.grad_tensors(grads[1:]), parts, norm_parts, ws, accumulate=True)
    assert float(parts) == pytest.approx(float(sum_sq), rel=1e-13) and float(norm_parts) == pytest.approx(float(norm), rel=1e-7)


def test_more_tensors_than_the_workspace_has_sums_for():
    """50 tables of 48 tensors, each with more pieces than a launch has workgroups: sums are folded on the way."""
    piece = 8192
    one = torch.ones(50 * piece, device=DEV)
    tensors = fb.grad_tensors(50 * 48 * [one])
    sum_sq, norm, _ = _scalars()
    ws = _ws()
    for _ in range(2):
        fb.fopd_grad_norm(tensors, sum_sq, norm, ws)
        assert float(sum_sq) == 50 * 48 * 50 * piece                         # (whole numbers: exact)
    fb.fopd_grad_norm(tensors, sum_sq, norm, ws, accumulate=True)
    assert float(sum_sq) == 2 * 50 * 48 * 50 * piece


def test_same_bits_each_time_and_in_a_captured_graph():
    grads = _tensors([(123, 457), (70001,), (5,)], [torch.float32, torch.bfloat16, torch.float32], seed=4)
    outs = [torch.empty_like(g) for g in grads]
    tensors, ws = fb.grad_tensors(grads, outs), _ws()
    sum_sq, norm, coef = _scalars()

    def both():
        fb.fopd_grad_norm(tensors, sum_sq, norm, ws)
        fb.fopd_grad_clip(tensors, sum_sq, 1.0, EPS, coef)

    both()
    first = [t.clone() for t in [sum_sq, norm, coef] + outs]
    both()
    assert all(torch.equal(a, b) for a, b in zip(first, [sum_sq, norm, coef] + outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    del tensors                                                              # (a captured launch keeps its own list)
    for seed in (5, 6, 7):
        for g, n in zip(grads, _tensors([g.shape for g in grads], [g.dtype for g in grads], seed=seed)):
            g.copy_(n)
        for t in [sum_sq, norm, coef] + outs:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        _check(grads, outs, [_f64(g) for g in grads], 1.0, sum_sq, norm, coef)


def test_entries_past_32_bit_offsets():
    """2^31 + 10 bf16 entries, one in front and one behind that are not zero."""
    g = torch.zeros((1 << 31) + 10, dtype=torch.bfloat16, device=DEV)
    g[3] = 3.0
    g[-2] = 4.0
    tensors = fb.grad_tensors([g])
    sum_sq, norm, coef = _scalars()
    fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
    assert float(norm) == 5.0
    fb.fopd_grad_clip(tensors, sum_sq, 2.5, 0.0, coef)
    assert float(g[3]) == 1.5 and float(g[-2]) == 2.0 and float(g[-1]) == 0.0


@pytest.mark.parametrize("most", [0.0, 1.0, float("inf")])
@pytest.mark.parametrize("place", ["in_place", "out"])
def test_zero_gradients_stay_zero_for_any_bound(most, place):
    grads = [torch.zeros(5000, device=DEV), torch.zeros(3, dtype=torch.bfloat16, device=DEV)]
    outs = grads if place == "in_place" else [torch.full_like(g, 7.0) for g in grads]
    tensors = fb.grad_tensors(grads, outs)
    for eps in (0.0, EPS):
        sum_sq, norm, coef = _scalars()
        fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
        fb.fopd_grad_clip(tensors, sum_sq, most, eps, coef)
        assert float(norm) == 0.0 and float(coef) == oo.grad_clip([_f64(g) for g in grads], most, eps)[2]
        assert all(bool((o == 0.0).all()) for o in outs)


def test_a_bound_of_zero_and_none_at_all():
    grads = [torch.randn(5000, generator=torch.Generator().manual_seed(1)).to(DEV)]
    outs = [torch.full_like(grads[0], 7.0)]
    tensors = fb.grad_tensors(grads, outs)
    sum_sq, norm, coef = _scalars()
    fb.fopd_grad_norm(tensors, sum_sq, norm, _ws())
    fb.fopd_grad_clip(tensors, sum_sq, 0.0, 0.0, coef)
    assert float(coef) == 0.0 and bool((outs[0] == 0.0).all())
    fb.fopd_grad_clip(tensors, sum_sq, float("inf"), 0.0, coef)
    assert float(coef) == 1.0 and torch.equal(outs[0], grads[0])
