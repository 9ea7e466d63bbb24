"""Verification of drafted tokens against the float64 oracle, and the step from a draft to clipped gradients."""

import math

import numpy as np
import pytest
import torch

from oracle import fopd_oracle as orc
from oracle import operators_oracle as oo
from paper_2605_17862_amd import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = {"f32": (torch.float32, fb.FOPD_F32, 4), "bf16": (torch.bfloat16, fb.FOPD_BF16, 8)}
# A decision is compared where its two sides are further apart than 32-bit arithmetic can be off: the bound of
# verify_logp_tolerance for either side is under 6e-5 at these sizes.
MARGIN = 2e-4


def _workspace(n):
    ws = torch.empty(n + 256, dtype=torch.uint8, device=DEV)
    off = (-ws.data_ptr()) % 256
    ws = ws[off:off + n]
    fb.fopd_workspace_init(ws)
    return ws


class Batch:
    """Inputs of a call, in a padded batch or (ragged) with rows of its samples in any place and unused rows between them."""

    def __init__(self, B, K, V, kind="bf16", seed=0, ragged=False, draft=True, taus=(1.0,), spread=3.0, away=0.5, lens=None, gap=0):
        dtype, self.dt, per = KINDS[kind]
        g = torch.Generator().manual_seed(seed * 1000 + B + K + V)
        self.B, self.K, self.V = B, K, V
        rs = np.random.RandomState(seed + 7)
        self.lens = np.array(lens if lens is not None else [rs.randint(0, K + 1) if ragged else K for _ in range(B)], dtype=np.int32)
        if gap:
            order, at, self.first = rs.permutation(B), gap, np.zeros(B, np.int64)
            for i in order:
                self.first[i] = at
                at += int(self.lens[i]) + 1 + gap
            self.R, self.row_begin = at, torch.from_numpy(self.first).to(DEV)
        else:
            self.R, self.first, self.row_begin = B * (K + 1), np.arange(B, dtype=np.int64) * (K + 1), None
        self.ld, self.ldd, self.lde = ((V + p - 1) // p * p + e for p, e in ((per, 0), (per, per), (4, 4)))
        z = torch.randn(self.R, V, generator=g) * spread
        zq = z + torch.randn(self.R, V, generator=g) * away
        self.target = torch.full((self.R, self.ld), float("nan"), dtype=dtype, device=DEV)
        self.target[:, :V] = z.to(dtype).to(DEV)
        self.draft = None
        if draft:
            self.draft = torch.full((self.R, self.ldd), float("nan"), dtype=dtype, device=DEV)
            self.draft[:, :V] = zq.to(dtype).to(DEV)
        self.taus = torch.tensor([taus[i % len(taus)] for i in range(B)])
        row_tau = torch.ones(self.R)
        for i in range(B):
            row_tau[self.first[i]:self.first[i] + self.lens[i] + 1] = max(float(self.taus[i]), 0.05)
        race = torch.empty(self.R, V).exponential_(1.0, generator=g).clamp_(min=1e-30).log_()
        self.ids = torch.argmax(zq.to(dtype).float() / row_tau[:, None] - race, dim=1).to(torch.int32).to(DEV)
        self.u = torch.rand(self.R, generator=g).to(DEV)
        self.noise = torch.empty(B, self.lde).exponential_(1.0, generator=g).clamp_(min=1e-30).to(DEV)
        self.temperature = self.taus.to(DEV)
        self.lens_d = torch.from_numpy(self.lens).to(DEV)
        self.greedy_call = False
        self.outs()
        self.ws = _workspace(fb.fopd_verify_workspace_bytes(self.R, V, B))

    def outs(self):
        self.n = torch.full((self.B,), -9, dtype=torch.int32, device=DEV)
        self.out_ids = torch.full((self.R,), -9, dtype=torch.int32, device=DEV)
        self.out_logp = torch.full((self.R,), 9.0, device=DEV)
        self.out_mask = torch.full((self.R,), 9, dtype=torch.uint8, device=DEV)

    def run(self, ws=None):
        rnd = (None, None) if self.greedy_call else (self.u, self.noise)
        fb.fopd_verify_draft(self.target, self.draft, self.dt, self.R, self.V, self.ld, self.ldd, self.ids, self.row_begin,
                             self.lens_d, self.B, self.K, self.temperature, rnd[0], rnd[1], self.lde, self.n, self.out_ids,
                             self.out_logp, self.out_mask, self.ws if ws is None else ws)

    def results(self):
        return [t.clone() for t in (self.n, self.out_ids, self.out_logp, self.out_mask)]

    def check(self, flags=0, at_least=0.9):
        V = self.V
        z = self.target[:, :V].double().cpu().numpy()
        zq = None if self.draft is None else self.draft[:, :V].double().cpu().numpy()
        noise = None if self.greedy_call else self.noise[:, :V].double().cpu().numpy()
        taus = self.taus.double().numpy()
        want = oo.verify(z, zq, self.ids.cpu().numpy(), self.first, self.lens, taus, self.u.double().cpu().numpy(), noise)
        n, ids, lp, mask = (t.cpu().numpy() for t in (self.n, self.out_ids, self.out_logp, self.out_mask))
        seen, compared = np.zeros(self.R, bool), 0
        for i, w in enumerate(want):
            r0, a = int(self.first[i]), w["kept"]
            last = self.K if self.row_begin is None else int(self.lens[i])
            seen[r0:r0 + last + 1] = True
            if w["margin"] < MARGIN:
                continue
            compared += 1
            assert n[i] == a, (i, n[i], w)
            assert (ids[r0:r0 + a] == self.ids.cpu().numpy()[r0:r0 + a]).all() and (mask[r0:r0 + a] == 1).all()
            if w["token"] is None:
                assert ids[r0 + a] == -1 and mask[r0 + a] == 0 and math.isnan(lp[r0 + a])
            else:
                assert ids[r0 + a] == w["token"] and mask[r0 + a] == 1, (i, ids[r0 + a], w)
            behind = slice(r0 + a + 1, r0 + last + 1)
            assert (ids[behind] == -1).all() and (mask[behind] == 0).all() and (lp[behind] == 0).all()
            tau = 0.0 if self.greedy_call else float(taus[i])
            for j, l in enumerate(w["logps"]):
                tol = oo.verify_logp_tolerance(z[r0 + j], int(ids[r0 + j]), tau)
                assert abs(lp[r0 + j] - l) <= tol, (i, j, lp[r0 + j], l, tol)
        assert compared >= at_least * self.B
        assert (ids[~seen] == -9).all() and (lp[~seen] == 9.0).all() and (mask[~seen] == 9).all()
        assert fb.fopd_workspace_status(self.ws)[1] == flags
        return want


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,K,V", [(1, 0, 1), (1, 1, 2), (3, 2, 7), (5, 4, 64), (33, 3, 1000), (7, 9, 2049), (64, 1, 4096), (2, 70, 300), (1, 4, 33001)])
def test_against_the_oracle(B, K, V, draft, kind):
    b = Batch(B, K, V, kind, draft=draft, taus=(0.7, 1.0, 1.6))
    b.run()
    b.check(at_least=0.7 if B < 4 else 0.9)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("gap", [0, 3])
def test_ragged_lengths_mixed_temperatures_and_rows_in_any_place(kind, draft, gap):
    b = Batch(41, 6, 515, kind, seed=3, ragged=True, draft=draft, taus=(0.6, 0.0, 1.0, 2.5), gap=gap)
    b.run()
    want = b.check()
    assert len({w["kept"] for w in want}) > 2              # (of the oracle alone: the batch has drafts cut at several places)


@pytest.mark.parametrize("B,K,V", [(2, 3, 151936), (30, 5, 32000), (1, 2, 262145)])
def test_vocabularies_of_models(B, K, V):
    b = Batch(B, K, V, "bf16", seed=5, taus=(0.7,))
    b.run()
    b.check(at_least=0.5 if B < 4 else 0.9)


def test_many_samples():
    b = Batch(3000, 1, 40, "f32", seed=6, ragged=True, taus=(1.0, 0.0))
    b.run()
    b.check()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_greedy_calls_take_no_variates_and_the_first_of_equals(kind):
    b = Batch(20, 4, 300, kind, seed=7, draft=True)
    b.target[:, :300] = torch.round(b.target[:, :300].float()).to(b.target.dtype)          # many equal largest entries
    best = b.target[:, :300].float().cpu().numpy().argmax(axis=1).astype(np.int32)
    ids = best.copy()
    ids[::3] = (ids[::3] + 1) % 300
    b.ids = torch.from_numpy(ids).to(DEV)
    b.greedy_call, b.temperature = True, None
    b.run()
    b.check(at_least=1.0)
    full = b.results()
    b.greedy_call, b.temperature, b.taus = False, torch.zeros(20, device=DEV), torch.zeros(20)
    b.noise.fill_(float("nan"))
    b.u.fill_(float("nan"))
    b.draft.fill_(float("nan"))
    b.outs()
    b.run()
    assert all(torch.equal(x, y) for x, y in zip(full, b.results()))


def test_no_lengths_and_no_temperature_mean_all_of_them_at_one():
    b = Batch(9, 3, 200, "f32", seed=8)
    b.run()
    full = b.results()
    b.lens_d = b.temperature = None
    b.outs()
    b.run()
    assert all(torch.equal(x, y) for x, y in zip(full, b.results()))


def test_without_drafts_it_draws_a_token_from_each_row():
    b = Batch(50, 0, 333, "bf16", seed=9, taus=(0.8,))
    b.ids = b.u = None
    b.run()
    b.ids, b.u = torch.zeros(50, dtype=torch.int32, device=DEV), torch.zeros(50, device=DEV)
    b.check()


@pytest.mark.parametrize("low", [float("-inf"), -3.3895313892515355e38])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_masked_entries_and_rows_of_nothing_else(low, kind):
    b = Batch(12, 3, 700, kind, seed=10, taus=(0.9,), away=0.2)
    keep = torch.rand(b.R, 700, generator=torch.Generator().manual_seed(1)).to(DEV) < 0.02
    keep[:, 5] = True
    b.target[:, :700] = torch.where(keep, b.target[:, :700], torch.full_like(b.target[:, :700], low))
    b.draft[:, :700] = torch.where(keep, b.draft[:, :700], torch.full_like(b.draft[:, :700], low))
    b.ids[:] = 5
    b.target[4 * 2 + 0, :700] = low                                        # the first row of sample 2
    b.target[4 * 7 + 3, :700] = low                                        # the last row of sample 7
    b.target[4 * 9 + 1, :650] = low                                        # a row that starts with nothing
    b.run()
    want = b.check(flags=16 if low == float("-inf") else 0)
    assert (want[2]["token"] is None) == (low == float("-inf"))            # all entries equal is a distribution, none is not


def test_rows_that_are_no_distribution():
    b = Batch(10, 3, 100, "f32", seed=11, away=0.0)
    b.u.fill_(0.0)                                                         # everything is kept where it can be
    b.target[4 * 1 + 1, 17] = float("nan")
    b.target[4 * 2 + 2, 99] = float("inf")
    b.target[4 * 3 + 3, 0] = float("nan")                                  # the row of the token after a whole draft
    b.draft[4 * 4 + 0, 3] = float("nan")
    b.draft[4 * 5 + 3, 3] = float("nan")                                   # not read
    b.run()
    want = b.check(flags=16, at_least=0.5)
    assert [w["kept"] for w in want[1:6]] == [1, 2, 3, 0, 3] and [w["token"] is None for w in want[1:6]] == [True] * 4 + [False]


def test_rows_behind_the_first_rejection_do_not_matter():
    b = Batch(6, 4, 100, "f32", seed=12)
    b.u[:] = 0.0
    b.u[1::5] = 2.0                                                        # draft 1 of every sample is refused
    b.target.view(6, 5, -1)[:, 2:] = float("nan")
    b.draft.view(6, 5, -1)[:, 2:] = float("nan")
    b.ids.view(6, 5)[:, 2:] = -5
    b.run()
    assert b.n.tolist() == [1] * 6 and fb.fopd_workspace_status(b.ws) == (0, 0)
    assert b.out_mask.view(6, 5).tolist() == 6 * [[1, 1, 0, 0, 0]]


def test_bad_temperatures_ids_and_places():
    b = Batch(6, 2, 90, "f32", seed=13, taus=(1.0,), away=0.0)
    b.u.fill_(0.0)
    b.taus = torch.tensor([1.0, -1.0, float("nan"), 1.0, 1.0, float("inf")])
    b.temperature = b.taus.to(DEV)
    b.run()
    assert b.n.tolist() == [2, 0, 0, 2, 2, 2] or b.n.tolist() == [2, 0, 0, 2, 2, 0]
    assert b.out_mask.view(6, 3)[1].tolist() == [0, 0, 0] and math.isnan(float(b.out_logp[3]))
    assert fb.fopd_workspace_status(b.ws) == (12, 16)
    # ids
    b = Batch(5, 2, 90, "f32", seed=13, away=0.0)
    b.u.fill_(0.0)
    b.ids[1] = 90
    b.ids[3] = -1
    b.ids[8] = 1 << 30                                                     # entry n of a sample is not read
    b.run()
    b.check(flags=1, at_least=0.6)
    assert b.n.tolist() == [1, 0, 2, 2, 2] and b.out_mask.sum() == 2 + 1 + 3 * 3
    # lengths in a padded batch
    b = Batch(4, 2, 90, "f32", seed=14, away=0.0)
    b.u.fill_(0.0)
    b.lens_d = torch.tensor([2, 3, -1, 0], dtype=torch.int32, device=DEV)
    b.run()
    assert b.n.tolist() == [2, 0, 0, 0] and b.out_mask.view(4, 3).tolist() == [[1, 1, 1], [0, 0, 0], [0, 0, 0], [1, 0, 0]]
    assert b.out_ids.view(4, 3)[1].tolist() == [-1, -1, -1] and fb.fopd_workspace_status(b.ws) == (7, 2)
    # rows that are not there
    b = Batch(5, 2, 90, "f32", seed=15, away=0.0, gap=1)
    b.u.fill_(0.0)
    first = b.first.copy()
    first[0], first[1], first[2], first[3] = -1, b.R - 2, 1 << 40, -(1 << 40)
    b.row_begin = torch.from_numpy(first).to(DEV)
    b.run()
    assert b.n.tolist() == [0, 0, 0, 0, 2] and fb.fopd_workspace_status(b.ws) == (7, 2)
    touched = torch.nonzero(b.out_ids != -9)[:, 0].tolist()
    assert touched == list(range(int(first[4]), int(first[4]) + 3))


def test_variates_at_their_ends():
    b = Batch(4, 1, 60, "f32", seed=16, away=0.0)                          # the drafter is the target
    b.u[:] = 1.0 - 2.0 ** -24
    b.draft[:, :60] = b.target[:, :60]
    b.run()
    assert b.n.tolist() == [1] * 4
    b.u[:] = 1.0                                                           # refused with nothing left: drawn from the target
    b.outs()
    b.run()
    assert b.n.tolist() == [0] * 4
    p = torch.softmax(b.target[::2, :60].double(), 1)
    assert b.out_ids[::2].tolist() == (p / b.noise[:, :60].double()).argmax(dim=1).tolist()
    b.noise.fill_(float("nan"))
    b.outs()
    b.run()
    assert b.out_ids[::2].tolist() == [-1] * 4 and b.out_mask[::2].tolist() == [0] * 4
    assert fb.fopd_workspace_status(b.ws) == (12, 16)


def test_same_bits_each_time_on_another_stream_and_in_a_captured_graph():
    b = Batch(13, 4, 5000, "bf16", seed=17, ragged=True, taus=(0.7, 0.0))
    b.run()
    first = b.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.outs()
        b.run()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, b.results()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run()
    for seed in (18, 19, 20):
        other = Batch(13, 4, 5000, "bf16", seed=seed, taus=(0.7, 0.0), lens=b.lens)
        for name in ("target", "draft", "ids", "u", "noise"):
            getattr(b, name).copy_(getattr(other, name))
        b.n.fill_(-9), b.out_ids.fill_(-9), b.out_logp.fill_(9.0), b.out_mask.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        b.check()
        other.run()
        assert all(torch.equal(x, y) for x, y in zip(other.results(), b.results()))


def test_two_calls_at_once_with_a_workspace_each():
    one, two = Batch(9, 3, 9000, "bf16", seed=21), Batch(3, 7, 20000, "f32", seed=22)
    one.run(), two.run()
    want = one.results() + two.results()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, s in ((one, streams[0]), (two, streams[1])):
            with torch.cuda.stream(s):
                b.run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, one.results() + two.results()))


def test_from_a_draft_to_clipped_gradients():
    """A drafter's logits through the 4-bit projection, tokens drawn from them and verified, the loss on what was kept, its
    gradients through the projection, their norm and clipping: each step takes what the one before left in memory."""
    B, K, V, d = 6, 3, 1000, 192
    R = B * (K + 1)
    g = torch.Generator().manual_seed(30)
    weight = (torch.randn(V, d, generator=g) * (3.0 / d ** 0.5)).to(torch.bfloat16).to(DEV)
    hidden = torch.randn(R, d, generator=g).to(torch.bfloat16).to(DEV)
    packed = torch.empty(fb.fopd_mx4_bytes(V, d), dtype=torch.uint8, device=DEV)
    fb.fopd_mx4_quantize(weight, fb.FOPD_BF16, V, d, d, packed)
    draft = torch.empty(R, V, device=DEV)
    fb.fopd_mx4_logits(hidden, fb.FOPD_BF16, d, packed, R, V, d, draft, fb.FOPD_F32, V,
                       _workspace(fb.fopd_mx4_logits_workspace_bytes(R, V, d)))
    b = Batch(B, K, V, "f32", seed=31, taus=(1.0,))
    race = torch.empty(R, V).exponential_(1.0, generator=g).clamp_(min=1e-30).to(DEV)
    b.draft, b.ldd = draft, V
    b.ids = (draft - race.log()).argmax(dim=1).to(torch.int32)
    b.target = (hidden.float() @ weight.float().t()).contiguous()
    b.run()
    b.check()
    T = R
    lens = torch.full((B,), K + 1, dtype=torch.int32, device=DEV)
    lag = torch.zeros(B, dtype=torch.int32, device=DEV)
    teacher = (b.out_logp - 0.3).contiguous()
    loss, weights, logp, lse = (torch.empty(n, device=DEV) for n in (1, B, T, T))
    dh, dw = torch.empty(T, d, device=DEV), torch.empty(V, d, device=DEV)
    ws = _workspace(fb.fopd_lm_head_loss_workspace_bytes(T, V, d, B, 64))
    hp = (1.0, 1.0, 0.05, 0.1)
    fb.fopd_lm_head_loss_fwd_bwd(hidden, d, weight, d, T, V, d, b.out_ids, b.out_mask, b.out_logp, teacher, lens, lag, B, hp,
                                 None, None, None, 1.0, 64, loss, weights, logp, lse, dh, d, dw, d, False, ws,
                                 seq_lens_host=lens.cpu())
    assert fb.fopd_workspace_status(ws) == (0, 0)                          # ids of -1 are masked
    kept = b.out_mask.bool()
    # the verified tokens' log-probs are the student's: its own pass finds the same ones (the two sum the same fp32 products
    # in another order: d 2^-23 of the magnitudes' sum, 3 sqrt(d) at most here, and twice that for the two of them)
    assert float((logp[kept] - b.out_logp[kept]).abs().max()) <= 2 * 192 * 2.0 ** -23 * 40.0
    grads = [dw, dh]
    before = [t.double().cpu().numpy() for t in grads]
    tensors = fb.grad_tensors(grads)
    n = fb.fopd_grad_workspace_bytes()
    sum_sq, norm, coef = torch.empty(1, dtype=torch.float64, device=DEV), torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    fb.fopd_grad_norm(tensors, sum_sq, norm, _workspace(n))
    most = 0.5 * math.sqrt(sum((x ** 2).sum() for x in before))
    fb.fopd_grad_clip(tensors, sum_sq, most, 1e-6, coef)
    _, want_n, want_c, want = oo.grad_clip(before, float(np.float32(most)), float(np.float32(1e-6)))
    assert abs(float(norm) - want_n) <= 2.0 ** -23 * want_n and abs(float(coef) - want_c) <= 2.0 ** -23 * want_c
    for t, w in zip(grads, want):
        assert (np.abs(t.double().cpu().numpy() - w) <= 2.0 ** -22 * np.abs(w) + 2.0 ** -149).all()


def _likely(rows, V, kind, tau, shift, masked=None, low=-1e9):
    """Rows of one token of probability 1 - 1e-9 or so, the others spread over some 10 tau below; the first `masked` entries `low`."""
    dtype, dt, per = KINDS[kind]
    g = torch.Generator().manual_seed(rows + V)
    z = torch.rand(rows, V, generator=g) * -10.0 - 21.0 - math.log(V)
    at = torch.randint(masked or 0, V, (rows,), generator=g)
    z[torch.arange(rows), at] = 0.0
    z = z * tau + shift
    if masked:
        z[:, :masked] = low
    ld = (V + per - 1) // per * per
    target = torch.full((rows, ld), float("nan"), dtype=dtype, device=DEV)
    target[:, :V] = z.to(dtype).to(DEV)
    return target, at, ld


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(3, 70), (5, 20011), (600, 5003)])
@pytest.mark.parametrize("tau,shift,masked,low", [
    (1.0, 0.0, 0, 0.0), (0.05, 3.0, 0, 0.0), (1.0, 100.0, 0, 0.0), (1.0, 1000.0, 0, 0.0), (0.6, 1000.0, 0, 0.0), (1.0, 5.0, 0.6, float("-inf")),
    (1.0, -150.0, 0, 0.0), (1.0, -1000.0, 0, 0.0), (0.1, -12.0, 0, 0.0),
    (1.0, 2.0, 0.6, -3.3895313892515355e38), (0.7, -120.0, 0.6, -1e9), (1.0, 0.0, 0.3, -10000.0)])
def test_log_probs_keep_their_digits_wherever_the_logits_lie(tau, shift, masked, low, rows, V, kind):
    target, at, ld = _likely(rows, V, kind, tau, shift, int(masked * V), low)
    taus = torch.full((rows,), tau, device=DEV)
    noise = torch.ones(rows, (V + 3) // 4 * 4, device=DEV)
    n, ids = (torch.full((rows,), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    logp, mask = torch.full((rows,), 9.0, device=DEV), torch.full((rows,), 9, dtype=torch.uint8, device=DEV)
    ws = _workspace(fb.fopd_verify_workspace_bytes(rows, V, rows))
    fb.fopd_verify_draft(target, None, KINDS[kind][1], rows, V, ld, ld, None, None, None, rows, 0, taus, None, noise, noise.shape[1],
                         n, ids, logp, mask, ws)
    assert fb.fopd_workspace_status(ws) == (0, 0)
    z = target[:, :V].double().cpu().numpy() / float(taus[0])
    s = z - z.max(axis=1, keepdims=True)
    assert (ids.cpu().numpy() == at.numpy()).all() and (mask == 1).all()
    s[np.arange(rows), at.numpy()] = -math.inf
    others = np.exp(s).sum(axis=1)                                         # (the bf16 ones near 1000 are 4 apart: ties among them)
    assert others.max() < 1e-2
    # a term's exponent t has five roundings relative to itself (log2 e, its division by tau, the multiply-add, and the difference and the
    # product where pieces meet); up to four exponentials of one unit in the last place (2^-23) multiply up, with as many
    # products; V / 256 + 64 additions; log1p and the result
    far = np.where(np.exp(s) > 0, np.abs(s), 0.0).max()
    tol = 2.0 ** -24 * (5.0 * far + 8.0 + 4.0 + V / 256 + 64 + 2.0)
    want = -np.log1p(others)
    off = np.abs(logp.double().cpu().numpy() - want)
    assert (off <= tol * np.abs(want)).all(), (off / np.maximum(np.abs(want), 1e-300)).max()


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("shift,taus", [(-150.0, (0.7, 1.0, 0.0)), (-9.0, (0.1, 0.2)), (-1000.0, (1.6,))])
def test_logits_far_below_zero(shift, taus, draft):
    b = Batch(21, 4, 5003, "f32", seed=41, draft=draft, taus=taus)
    b.target += shift
    if draft:
        b.draft += shift
    b.run()
    b.check(at_least=0.7)


def test_smaller_batches_in_the_workspace_of_a_larger_one():
    """The batch shrinks as its samples end, and the workspace stays."""
    V = 9000
    n = fb.fopd_verify_workspace_bytes(2048, V, 256)
    guarded = _workspace(n + 4096)
    ws = guarded[:n]
    guarded[n:] = 77
    for B, K in ((255, 7), (128, 7), (127, 7), (16, 3), (1, 0)):
        b = Batch(B, K, V, "bf16", seed=42, taus=(0.7,))
        b.run(ws)
        b.ws = ws
        b.check(at_least=0.7 if B > 1 else 0.0)
    assert bool((guarded[n:] == 77).all())


@pytest.mark.parametrize("V", [5000, 40001, 151936])
@pytest.mark.parametrize("B", [1, 3, 70])
def test_a_race_over_many_pieces_that_nobody_wins(B, V):
    """The drafter is the target and the draft is refused all the same: the last workgroup races for the target's own row."""
    b = Batch(B, 1, V, "f32", seed=43, away=0.0, taus=(0.8,))
    b.draft[:, :V] = b.target[:, :V]
    b.u[:] = 1.0
    for _ in range(3):
        b.outs()
        b.run()
        assert b.n.tolist() == [0] * B
        z = b.target[::2, :V].double() / b.temperature.double()[:, None]
        score = torch.log_softmax(z, 1) - b.noise[:, :V].double().log()
        first, second = score.topk(2, dim=1).values.unbind(1)
        sure = first - second > MARGIN
        assert int(sure.sum()) >= 0.9 * B
        assert torch.equal(b.out_ids[::2][sure].long(), score.argmax(dim=1)[sure])
        assert b.out_mask.tolist() == B * [1, 0] and fb.fopd_workspace_status(b.ws) == (0, 0)


def test_the_largest_vocabulary():
    """2^31 - 512 entries, whose last places are as far as 32 bits go."""
    V = (1 << 31) - 512 - 3                                                # (entries behind the last whole vector)
    ld = (V + 7) // 8 * 8
    target = torch.full((1, ld), float("-inf"), dtype=torch.bfloat16, device=DEV)
    places = [0, 12345, (1 << 30) + 1, V - 300, V - 2, V - 1]
    z = [1.0, 2.0, 0.5, 1.5, 2.5, 1.0]
    target[0, places] = torch.tensor(z, dtype=torch.bfloat16, device=DEV)
    noise = torch.ones(1, ld, device=DEV)
    n, ids = (torch.full((1,), -9, dtype=torch.int32, device=DEV) for _ in range(2))
    logp, mask = torch.full((1,), 9.0, device=DEV), torch.full((1,), 9, dtype=torch.uint8, device=DEV)
    ws = _workspace(fb.fopd_verify_workspace_bytes(1, V, 1))
    p = np.exp(z) / np.exp(z).sum()
    for first in range(len(places)):                                       # each of them wins once
        noise[0, places] = 1.0
        noise[0, places[first]] = 0.01
        fb.fopd_verify_draft(target, None, fb.FOPD_BF16, 1, V, ld, ld, None, None, None, 1, 0, None, None, noise, ld, n, ids, logp, mask, ws)
        assert (int(n), int(ids), int(mask)) == (0, places[first], 1)
        assert abs(float(logp) - math.log(p[first])) <= 2.0 ** -20         # (six terms)
    fb.fopd_verify_draft(target, None, fb.FOPD_BF16, 1, V, ld, ld, None, None, None, 1, 0, None, None, None, 0, n, ids, logp, mask, ws)
    assert int(ids) == V - 2 and fb.fopd_workspace_status(ws) == (0, 0)


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("tau", [1.0, 1e-20, 1e-37, 5e-39, 4e-39, 1e-42, 2.0 ** -149])
def test_the_smallest_temperatures_leave_the_largest_entries(tau, draft):
    """From some size down p is 1 / n at the n largest entries and 0 elsewhere; the temperature's inverse need not be a number of the type."""
    b = Batch(12, 2, 5003, "f32", seed=44, draft=draft, taus=(tau,))
    z = torch.round(b.target[:, :5003] * 2.0)
    b.target[:, :5003] = z
    b.target[4, :5003] -= z[4].max()                                       # (a largest entry of 0)
    if draft:
        b.draft[:, :5003] = z + torch.round(torch.randn(z.shape, generator=torch.Generator().manual_seed(2)).to(DEV) * 0.6)
    b.ids = z.argmax(dim=1).to(torch.int32)
    b.ids[::5] = 7
    b.run()
    b.check(at_least=0.9)


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("tau", [-1.0, -1e-45, float("nan"), float("inf"), float("-inf")])
def test_a_temperature_that_is_none_ends_its_sample_before_the_first_row(tau, draft):
    b = Batch(3, 2, 90, "f32", seed=45, draft=draft, away=0.0)
    b.u.fill_(0.0)
    b.taus = torch.tensor([1.0, tau, 1.0])
    b.temperature = b.taus.to(DEV)
    b.run()
    assert b.n.tolist() == [2, 0, 2] and fb.fopd_workspace_status(b.ws) == (12, 16)
    ids, logp, mask = b.out_ids.view(3, 3), b.out_logp.view(3, 3), b.out_mask.view(3, 3)
    assert ids[1].tolist() == [-1, -1, -1] and mask.tolist() == [[1, 1, 1], [0, 0, 0], [1, 1, 1]]
    assert math.isnan(float(logp[1, 0])) and logp[1, 1:].tolist() == [0.0, 0.0]
    assert bool(torch.isfinite(logp[[0, 2]]).all()) and torch.equal(ids[[0, 2], :2], b.ids.view(3, 3)[[0, 2], :2])


def test_verified_rollouts_and_the_loss_at_other_temperatures_than_one():
    """Verification gives log-probs at the sampling temperature; the loss forms its own at 1.  With behaviour log-probs at 1, from
    fopd_token_logprobs over the verified rows, a fresh sample (lag 0) has no drift."""
    B, K, V = 8, 3, 1500
    b = Batch(B, K, V, "bf16", seed=46, taus=(0.6, 0.7))
    b.run()
    b.check()
    T = b.R
    lens, lag = torch.full((B,), K + 1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    loss_ws = _workspace(fb.fopd_workspace_bytes(T, B))
    at_one, lse = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    fb.fopd_token_logprobs(b.target, b.dt, T, V, b.ld, b.out_ids, b.out_mask, at_one, lse, None, None, loss_ws)
    kept = b.out_mask.bool()
    z = b.target[:, :V].double()
    want = torch.log_softmax(z, 1).gather(1, b.out_ids.long().clamp(min=0)[:, None])[:, 0]
    assert float((at_one.double() - want)[kept].abs().max()) <= 1e-4
    assert float((b.out_logp.double() - want)[kept].abs().max()) > 1e-2   # (the two temperatures differ)
    teacher = (at_one - 0.3).contiguous()
    drift = {}
    for name, behav in (("at one", at_one), ("sampled", b.out_logp)):
        out = [torch.empty(B, dtype=dt, device=DEV) for dt in (torch.int32, torch.int32) + 6 * (torch.float32,)]
        agg, cu = torch.empty(3, device=DEV), torch.empty(B + 1, dtype=torch.int64, device=DEV)
        n_train, n_roll, d_roll, d_sup, ell, cover, cover_roll, fresh = out
        fb.fopd_freshness_score(at_one, behav, None, None, teacher, None, b.out_mask, lens, lag, T, B, (1.0, 1.0, 0.05, 0.1), cu,
                                n_train, n_roll, d_roll, d_sup, ell, cover, cover_roll, fresh, agg, loss_ws)
        drift[name] = d_roll.clone()
        assert n_train.tolist() == (b.n + 1).tolist()
    assert fb.fopd_workspace_status(loss_ws) == (0, 0)
    assert bool((drift["at one"] == 0.0).all()) and bool((drift["sampled"] != 0.0).all())
