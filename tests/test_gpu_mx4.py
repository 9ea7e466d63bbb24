"""4-bit blocks and the projection kept in them, against the float64 oracle."""

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo
from paper_2605_17862_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = {"f32": (torch.float32, fb.FOPD_F32, 4), "bf16": (torch.bfloat16, fb.FOPD_BF16, 8)}


def _matrix(R, d, kind, seed, spread=8, pitch=None):
    """Rows of different size, zeros and small entries among them, in a padded buffer whose padding is NaN."""
    dtype, _, per = KINDS[kind]
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, d, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, (R, 1), generator=g).float())
    x[torch.rand(R, d, generator=g) < 0.1] *= 2.0 ** -6
    x[torch.rand(R, d, generator=g) < 0.05] = 0.0
    ld = pitch or (d + per - 1) // per * per
    buf = torch.full((R, ld), float("nan"), dtype=dtype, device=DEV)
    buf[:, :d] = x.to(dtype).to(DEV)
    return buf, buf[:, :d].double().cpu().numpy()


def _pack(buf, kind, R, d):
    packed = torch.full((fb.fopd_mx4_bytes(R, d),), 255, dtype=torch.uint8, device=DEV)
    fb.fopd_mx4_quantize(buf, KINDS[kind][1], R, d, buf.shape[1], packed)
    return packed


def _workspace(n):
    ws = torch.empty(n + 256, dtype=torch.uint8, device=DEV)
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("R,d,pitch", [(1, 1, None), (1, 32, None), (3, 31, None), (5, 33, 64), (64, 256, None), (65, 257, 320), (130, 500, None), (200, 1024, None),
                                       (17, 2008, 2048)])
def test_blocks_are_the_oracles_byte_for_byte(kind, R, d, pitch):
    buf, x = _matrix(R, d, kind, seed=R + d, pitch=pitch)
    packed = _pack(buf, kind, R, d)
    want = oo.mx4_packed(x).reshape(-1, 8704)
    got = packed.cpu().numpy().reshape(-1, 8704)
    # (-0 and 0 are the same value; what the sign of a zero is, is not fixed)
    for half in (lambda b: b & 15, lambda b: b >> 4):
        one, other = (np.where(half(b[:, :8192]) == 8, 0, half(b[:, :8192])) for b in (got, want))
        assert (one == other).all()
    assert (got[:, 8192:] == want[:, 8192:]).all()
    values = oo.mx4_blocks(x)[2]
    for out_kind in ("f32", "bf16"):
        dtype, dt, per = KINDS[out_kind]
        ldo = (d + per - 1) // per * per + per
        out = torch.full((R, ldo), 7.0, dtype=dtype, device=DEV)
        fb.fopd_mx4_dequantize(packed, R, d, out, dt, ldo)
        assert (out[:, :d].double().cpu().numpy() == values).all()
        assert bool((out[:, d:] == 7.0).all())                       # columns behind the last are not written


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_every_border_between_two_values(kind):
    """Each midpoint and its neighbours, at the ends of the range of the shared power and where it is clamped."""
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    eps = 2.0 ** -7 if kind == "bf16" else 2.0 ** -23
    row = [4.0] + [m * f for m in mids for f in (1.0, 1.0 - eps, 1.0 + eps)] + [-m for m in mids] + [7.5, -6.5, 0.0]
    x = torch.tensor([row + [0.0] * (32 - len(row))], dtype=torch.float64)
    scales = [2.0 ** e for e in (-126, -125, -20, 0, 1, 60, 124)]
    x = torch.cat([x * s for s in scales] + [torch.zeros(1, 32, dtype=torch.float64), torch.full((1, 32), 2.0 ** -130, dtype=torch.float64),
                                             torch.full((1, 32), -3.0e38, dtype=torch.float64)])
    buf = x.to(KINDS[kind][0]).to(DEV).contiguous()
    R = buf.shape[0]
    packed = _pack(buf, kind, R, 32)
    out = torch.empty(R, 32, device=DEV)
    fb.fopd_mx4_dequantize(packed, R, 32, out, fb.FOPD_F32, 32)
    assert (out.double().cpu().numpy() == oo.mx4_blocks(buf.double().cpu().numpy())[2]).all()


def test_a_row_that_is_nan_among_many():
    h, _ = _matrix(1300, 300, "bf16", seed=9)
    h[1100, 299] = float("inf")
    w, _ = _matrix(6000, 300, "bf16", seed=10)
    w[5999, 0] = float("nan")
    z = torch.zeros(1300, 6000, device=DEV)
    fb.fopd_mx4_logits(h, fb.FOPD_BF16, h.shape[1], _pack(w, "bf16", 6000, 300), 1300, 6000, 300, z, fb.FOPD_F32, 6000,
                       _workspace(fb.fopd_mx4_logits_workspace_bytes(1300, 6000, 300)))
    nan = torch.isnan(z)
    assert bool(nan[1100].all()) and bool(nan[:, 5999].all()) and int(nan.sum()) == 6000 + 1299


def test_infinities_and_nan_make_their_block_nan_and_no_other():
    buf, x = _matrix(70, 320, "bf16", seed=5)
    buf[3, 40] = float("inf")
    buf[66, 0] = float("nan")
    buf[69, 319] = float("-inf")
    packed = _pack(buf, "bf16", 70, 320)
    out = torch.empty(70, 320, device=DEV)
    fb.fopd_mx4_dequantize(packed, 70, 320, out, fb.FOPD_F32, 320)
    want = oo.mx4_blocks(buf.double().cpu().numpy())[2]
    assert np.isnan(want).sum() == 96
    assert np.array_equal(out.double().cpu().numpy(), want, equal_nan=True)
    # a product with such a row is NaN, the others are not touched by it
    w, wx = _matrix(100, 320, "bf16", seed=6)
    z = torch.zeros(70, 104, device=DEV)
    fb.fopd_mx4_logits(buf, fb.FOPD_BF16, 320, _pack(w, "bf16", 100, 320), 70, 100, 320, z, fb.FOPD_F32, 104,
                       _workspace(fb.fopd_mx4_logits_workspace_bytes(70, 100, 320)))
    nan = torch.isnan(z[:, :100])
    assert bool(nan[[3, 66, 69]].all()) and int(nan.sum()) == 300


def test_a_row_that_is_nan_among_few():
    """The same for the kernel of few rows, and a weight row that is NaN."""
    h, _ = _matrix(20, 300, "f32", seed=7)
    h[17, 299] = float("inf")
    w, _ = _matrix(130, 300, "bf16", seed=8)
    w[129, 0] = float("nan")
    z = torch.zeros(20, 136, device=DEV)
    fb.fopd_mx4_logits(h, fb.FOPD_F32, h.shape[1], _pack(w, "bf16", 130, 300), 20, 130, 300, z, fb.FOPD_F32, 136,
                       _workspace(fb.fopd_mx4_logits_workspace_bytes(20, 130, 300)))
    nan = torch.isnan(z[:, :130])
    assert bool(nan[17].all()) and bool(nan[:, 129].all()) and int(nan.sum()) == 130 + 19


def _logits(T, V, d, kind_h, kind, seed, h_pitch=None):
    hb, hx = _matrix(T, d, kind_h, seed, spread=2, pitch=h_pitch)
    wb, wx = _matrix(V, d, "bf16", seed + 1, spread=2)
    packed = _pack(wb, "bf16", V, d)
    dtype, dt, per = KINDS[kind]
    ld = (V + per - 1) // per * per + per
    z = torch.full((T + 1, ld), 7.0, dtype=dtype, device=DEV)
    ws = _workspace(fb.fopd_mx4_logits_workspace_bytes(T, V, d))
    args = (hb, KINDS[kind_h][1], hb.shape[1], packed, T, V, d, z, dt, ld, ws)
    fb.fopd_mx4_logits(*args)
    return z, hx, wx, args


def _check(z, hx, wx, T, V, d, kind):
    h, w = (torch.from_numpy(oo.mx4_blocks(m)[2]) for m in (hx, wx))
    want, size = h @ w.t(), h.abs() @ w.abs().t()
    # fp32 sums in any order: at most d additions of terms whose magnitudes add up to `size`, each off by at most a unit in the
    # last place; then the rounding to the result's type
    tol = d * 2.0 ** -23 * size + (2.0 ** -8 if kind == "bf16" else 2.0 ** -24) * want.abs() * 1.01
    off = (z[:T, :V].double().cpu() - want).abs()
    assert bool((off <= tol).all()), float((off / tol.clamp(min=1e-300)).max())
    assert bool((z[:T, V:] == 7.0).all()) and bool((z[T:] == 7.0).all())


@pytest.mark.parametrize("kind_h,kind", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 64, 256), (2, 65, 33), (15, 100, 300), (16, 1000, 512), (17, 130, 1024), (33, 255, 700),
                                   (64, 257, 256), (65, 64, 2000), (100, 300, 520), (255, 600, 257), (256, 256, 256), (257, 513, 300), (300, 1030, 1536),
                                   (1000, 777, 96), (1500, 4000, 64), (65, 50001, 33), (257, 25000, 300), (2049, 4100, 257),
                                   (1100, 6003, 513)])
def test_product_against_the_oracle(T, V, d, kind_h, kind):
    z, hx, wx, _ = _logits(T, V, d, kind_h, kind, seed=T + V)
    _check(z, hx, wx, T, V, d, kind)


@pytest.mark.parametrize("T,V,d,kind", [(1, 151936, 256, "bf16"), (40, 40000, 1024, "bf16"), (600, 30001, 520, "f32"), (2100, 20000, 300, "bf16")])
def test_product_of_many_tiles(T, V, d, kind):
    z, hx, wx, _ = _logits(T, V, d, "bf16", kind, seed=T)
    _check(z, hx, wx, T, V, d, kind)


@pytest.mark.parametrize("T,V,d", [(3, 1000, 512), (300, 5000, 768), (1100, 6003, 513)])
def test_product_twice_captured_and_on_another_stream_gives_the_same_bits(T, V, d):
    z, hx, wx, args = _logits(T, V, d, "bf16", "bf16", seed=9)
    first = z.clone()
    fb.fopd_mx4_logits(*args)
    assert torch.equal(z, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z.fill_(7.0)
        fb.fopd_mx4_logits(*args)
    side.synchronize()
    assert torch.equal(z, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fb.fopd_mx4_logits(*args)
    for seed in (1, 2, 3):
        hb, hx2 = _matrix(T, d, "bf16", seed, spread=2)
        args[0].copy_(hb)
        z.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        _check(z, hx2, wx, T, V, d, "bf16")
        replayed = z.clone()
        fb.fopd_mx4_logits(*args)
        assert torch.equal(z, replayed)


def test_two_products_at_once_with_a_workspace_each():
    one, other = (_logits(T, 3000, 512, "bf16", "f32", seed=s) for T, s in ((5, 1), (2300, 2)))
    torch.cuda.synchronize()
    want = [one[0].clone(), other[0].clone()]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (z, _, _, args), s in zip((one, other), streams):
            with torch.cuda.stream(s):
                fb.fopd_mx4_logits(*args)
    torch.cuda.synchronize()
    assert torch.equal(one[0], want[0]) and torch.equal(other[0], want[1])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 777, 20003])
@pytest.mark.parametrize("d,pitch", [(1, None), (77, 96), (1000, None), (1531, 1536)])
def test_few_rows_give_the_bits_they_have_among_more(V, d, pitch, kind):
    """Each sum is taken in one order, however many rows stand beside it and whether the rows are packed first."""
    h, _ = _matrix(20, d, kind, seed=V + d, pitch=pitch)
    h[2, d // 2] = float("inf")                                      # NaN results, in a row that few of the calls have
    h[3, :d] = 0.0
    h[5, d - 1] = float("nan")
    w, _ = _matrix(V, d, "bf16", seed=9, spread=2)
    packed, ld = _pack(w, "bf16", V, d), (V + 3) // 4 * 4
    rows = {}
    for T in (20, 16, 8, 6, 2, 1):
        rows[T] = torch.full((T, ld), 7.0, device=DEV)
        fb.fopd_mx4_logits(h, KINDS[kind][1], h.shape[1], packed, T, V, d, rows[T], fb.FOPD_F32, ld,
                           _workspace(fb.fopd_mx4_logits_workspace_bytes(T, V, d)))
    assert bool(torch.isnan(rows[20][[2, 5], :V]).all()) and not bool(torch.isnan(rows[20][[0, 1, 3, 4, 19]]).any())
    for T in (16, 8, 6, 2, 1):
        assert np.array_equal(rows[T].cpu().numpy(), rows[20][:T].cpu().numpy(), equal_nan=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,d", [(49, 32769, 1), (64, 33000, 256), (65, 40001, 257), (96, 32831, 800), (97, 33003, 513), (128, 32960, 1500), (127, 50001, 33),
                                   (129, 24577, 600), (160, 24700, 257), (150, 30001, 65)])
def test_product_of_some_rows_with_a_large_vocabulary(T, V, d, kind):
    z, hx, wx, _ = _logits(T, V, d, "bf16", kind, seed=T + V + d)
    _check(z, hx, wx, T, V, d, kind)


def test_product_of_some_rows_with_a_weight_that_no_cache_holds():
    T, V, d = 100, 151936, 1800
    h, hx = _matrix(T, d, "bf16", seed=3, spread=2)
    w = torch.randn(V, d, generator=torch.Generator(DEV).manual_seed(4), device=DEV).bfloat16()
    z = torch.full((T + 1, V + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    fb.fopd_mx4_logits(h, fb.FOPD_BF16, d, _pack(w, "bf16", V, d), T, V, d, z, fb.FOPD_BF16, V + 8,
                       _workspace(fb.fopd_mx4_logits_workspace_bytes(T, V, d)))
    at = np.unique(np.r_[0:130, V - 130:V, np.random.default_rng(0).integers(0, V, 500)])
    _check(torch.cat((z[:, at], z[:, V:]), 1), hx, w[at].double().cpu().numpy(), T, len(at), d, "bf16")


def test_some_rows_that_are_nan_captured_and_replayed():
    T, V, d = 70, 40000, 600
    z, _, _, args = _logits(T, V, d, "f32", "f32", seed=11)
    hb = args[0]
    hb[66, 599] = float("nan")
    want = torch.empty_like(z)
    fb.fopd_mx4_logits(*args)
    want.copy_(z)
    assert bool(torch.isnan(want[66, :V]).all()) and int(torch.isnan(want).sum()) == V
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fb.fopd_mx4_logits(*args)
    for _ in range(3):
        z[:T, :V] = 0.0
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(z.cpu().numpy(), want.cpu().numpy(), equal_nan=True)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,d", [(65, 16385, 300), (96, 17003, 513), (128, 16450, 257), (129, 21889, 96), (160, 22001, 520), (128, 16384, 200), (160, 21800, 257),
                                   (192, 27001, 130), (224, 22528, 300), (225, 22600, 300), (1024, 5632, 257), (1000, 5600, 96), (1030, 5888, 64)])
def test_product_either_side_of_the_kernels_borders(T, V, d, kind):
    z, hx, wx, _ = _logits(T, V, d, "bf16", kind, seed=T + V + d)
    _check(z, hx, wx, T, V, d, kind)
