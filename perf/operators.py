"""The operators around the loss pass, as cases that can be timed: drafting with a 4-bit projection, verifying the drafted
tokens, and the gradient norm with clipping that stands between the loss's gradients and the optimiser.

`own` chooses between the plain forms (elementary torch operations in 32 or 64 bits) and this library's entry points.  The
shapes are those of the repository's workloads: a vocabulary of 151,936 entries and a hidden size of 4096 (reasoning, tool
use, coding), 262,144 entries (the large vocabulary), 4096 entries in fp32 (tiny), and 32,000 entries between them.
"""

import functools
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6                          # what a clipping program adds to the norm

# op        verify    drafted tokens against the student's logits, with the next token from given random numbers
#           quantize  a matrix to 4-bit blocks, and the values that they hold back again (a checkpoint's round trip)
#           logits    hidden states times a projection kept in 4 bits
#           clip      global norm of a list of gradients, and the gradients scaled by it
# verify: B samples of up to K drafted tokens each, ragged lengths or all K, V entries, draft: the drafter's logits are at
# hand (else the tokens alone, as from an n-gram lookup), greedy: every so many samples one is decoded greedily (0: none)


def listed():
    return [
        # one rollout being decoded, five rows: latency
        dict(name="verify_one_rollout", op="verify", dtype="bf16", B=1, K=4, V=151936, ragged=False, draft=True, greedy=0),
        # the tiny configuration, fp32: launches are all there is
        dict(name="verify_tiny_f32", op="verify", dtype="f32", B=4, K=3, V=4096, ragged=True, draft=True, greedy=2),
        # a rollout server's batch with a drafter, every draft full length
        dict(name="verify_batch", op="verify", dtype="bf16", B=192, K=7, V=151936, ragged=False, draft=True, greedy=0),
        # the large vocabulary, drafts looked up in the prompt, of any length; every third sample greedy
        dict(name="verify_lookup", op="verify", dtype="bf16", B=37, K=5, V=262144, ragged=True, draft=False, greedy=3),
        # the student's output projection laid out for its drafter after a weight update
        dict(name="quantize_head", op="quantize", dtype="bf16", R=151936, d=4096),
        # hidden states of a few rollouts in fp32, a width that ends inside a block
        dict(name="quantize_hidden", op="quantize", dtype="f32", R=1037, d=2008),
        # one token drafted: the projection is read once
        dict(name="logits_one_token", op="logits", dtype="bf16", T=1, V=151936, d=4096),
        # one token drafted for each of a server's rollouts
        dict(name="logits_draft_step", op="logits", dtype="bf16", T=45, V=151936, d=4096),
        # whole rollouts scored under the 4-bit projection
        dict(name="logits_rollouts", op="logits", dtype="bf16", T=4096, V=151936, d=4096),
        # the tiny configuration's gradients
        dict(name="clip_tiny", op="clip", dtype="f32", kind="tiny", width=256, V=4096, layers=2),
        # gradient of the output projection in fp32 and of the norm in front of it
        dict(name="clip_head", op="clip", dtype="f32", kind="head", width=4096, V=151936, layers=0),
        # matrices and norms of several layers in bf16
        dict(name="clip_layers", op="clip", dtype="bf16", kind="layers", width=4096, V=0, layers=8),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["verify", "verify", "quantize", "logits", "logits", "clip"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if op == "verify":
        V = rng.choice([4096, 32000, 151936, 262144, _log_uniform(rng, 4096, 262144), _log_uniform(rng, 4096, 262144)])
        K = rng.randint(1, 9)
        most = int(2.3e8 / (V * (K + 1) * (2 if dtype == "f32" else 1)))
        return dict(op=op, dtype=dtype, B=_log_uniform(rng, 1, max(2, min(256, most))), K=K, V=V, ragged=rng.random() < 0.5,
                    draft=rng.random() < 0.7, greedy=rng.choice([0, 0, 2, 5]))
    if op == "quantize":
        d = rng.choice([4096, 64 * rng.randint(2, 64), 8 * rng.randint(16, 512)])
        return dict(op=op, dtype=dtype, R=_log_uniform(rng, 1, 151936 if dtype == "bf16" else 65536), d=d)
    if op == "logits":
        d = rng.choice([4096, 64 * rng.randint(8, 64), 8 * rng.randint(64, 512)])
        T = rng.choice([_log_uniform(rng, 1, 64), _log_uniform(rng, 1, 2048 if dtype == "f32" else 4096)])
        return dict(op=op, dtype=dtype, T=T, V=rng.choice([32000, 151936, _log_uniform(rng, 4096, 151936)]), d=d)
    kind = rng.choice(["head", "layers"])
    width = 8 * _log_uniform(rng, 16, 480) + rng.choice([0, 0, 1, 5])
    return dict(op=op, dtype=dtype, kind=kind, width=width, V=_log_uniform(rng, 4096, 151936) if kind == "head" else 0,
                layers=0 if kind == "head" else rng.randint(1, 8))


# ---- what does not depend on the seed ---------------------------------------------------------------------------


@functools.lru_cache(maxsize=64)
def _lens_of(B, K, V, ragged):
    rs = random.Random("%d %d %d" % (B, K, V))
    return tuple(rs.randint(0, K) if ragged else K for _ in range(B))


def _lens(case):
    return _lens_of(case["B"], case["K"], case["V"], case["ragged"])


def _is_greedy(case):
    return [case["greedy"] > 0 and i % case["greedy"] == case["greedy"] - 1 for i in range(case["B"])]


def _pitch(V, dtype):
    per = 4 if dtype == "f32" else 8
    return (V + per - 1) // per * per                                # rows are 16-byte aligned


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gradient_shapes(case):
    w = case["width"]
    if case["kind"] == "head":
        return [(case["V"], w), (w,)]
    if case["kind"] == "tiny":
        return [(case["V"], w), (w,)] + case["layers"] * [(w, w), (w,), (w,)]
    return case["layers"] * [(w, w), (2 * w, w), (w, 2 * w), (w,), (w,)] + [(w,)]


# ---- inputs -----------------------------------------------------------------------------------------------------


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 1000003 + 29)
    return dict(case=case, **{"verify": _prepare_verify, "quantize": _prepare_quantize, "logits": _prepare_logits,
                              "clip": _prepare_clip}[case["op"]](case, gen))


def _prepare_verify(case, gen):
    B, K, V, dtype = case["B"], case["K"], case["V"], _type(case)
    R, ld = B * (K + 1), _pitch(case["V"], case["dtype"])
    greedy = _is_greedy(case)
    s = dict(target=torch.zeros(R, ld, dtype=dtype, device=DEV), draft_ids=torch.empty(R, dtype=torch.int32, device=DEV),
             draft=torch.zeros(R, ld, dtype=dtype, device=DEV) if case["draft"] else None,
             draft_lens=torch.tensor(_lens(case), dtype=torch.int32, device=DEV),
             temperature=torch.tensor([0.0 if g else (0.7, 1.0, 0.6)[i % 3] for i, g in enumerate(greedy)], device=DEV))
    per_row = torch.where(s["temperature"] > 0, s["temperature"], torch.full_like(s["temperature"], 0.1)).repeat_interleave(K + 1)
    rows = max(K + 1, (1 << 27) // V)
    for a in range(0, R, rows):
        b = min(a + rows, R)
        # raw logits of a language model: N(0, 3^2) with 32 strongly preferred tokens a row; the drafter is a little off
        z = torch.randn(b - a, V, generator=gen, device=DEV).mul_(3.0)
        z.scatter_add_(1, torch.randint(0, V, (b - a, 32), generator=gen, device=DEV), torch.full((b - a, 32), 8.0, device=DEV))
        s["target"][a:b, :V] = z
        z.add_(torch.randn(b - a, V, generator=gen, device=DEV), alpha=0.4)
        if case["draft"]:
            s["draft"][a:b, :V] = z
            z = s["draft"][a:b, :V].float()
        race = torch.empty_like(z).exponential_(1.0, generator=gen).clamp_(min=1e-30).log_()
        s["draft_ids"][a:b] = torch.argmax(z / per_row[a:b, None] - race, dim=1).to(torch.int32)
    s["accept_u"] = torch.rand(R, generator=gen, device=DEV)
    s["noise"] = torch.empty(B, ld, device=DEV).exponential_(1.0, generator=gen).clamp_(min=1e-30)
    s.update(n_accepted=torch.empty(B, dtype=torch.int32, device=DEV), out_ids=torch.empty(R, dtype=torch.int32, device=DEV),
             out_logp=torch.empty(R, device=DEV), out_mask=torch.empty(R, dtype=torch.uint8, device=DEV))
    return s


def _pad_columns(x, ld):
    if x.shape[1] == ld:
        return x
    y = torch.zeros(x.shape[0], ld, dtype=x.dtype, device=x.device)
    y[:, :x.shape[1]] = x
    return y


def _prepare_quantize(case, gen):
    R, d, dtype = case["R"], case["d"], _type(case)
    scale = torch.rand(R, 1, generator=gen, device=DEV).mul_(4.0).exp2_()          # rows of different size
    x = torch.randn(R, d, generator=gen, device=DEV).mul_(scale)
    return dict(x=_pad_columns(x.to(dtype), _pitch(d, case["dtype"])),
                values=torch.zeros(R, _pitch(d, "bf16"), dtype=torch.bfloat16, device=DEV))


def _prepare_logits(case, gen):
    T, V, d = case["T"], case["V"], case["d"]
    weight = torch.empty(V, _pitch(d, "bf16"), dtype=torch.bfloat16, device=DEV).zero_()
    rows = max(1, (1 << 27) // d)
    for a in range(0, V, rows):                                      # a projection as a 4-bit checkpoint holds it
        b = min(a + rows, V)
        weight[a:b, :d] = _to_blocks(torch.randn(b - a, d, generator=gen, device=DEV).mul_(3.0 / d ** 0.5))
    hidden = torch.randn(T, d, generator=gen, device=DEV).to(torch.bfloat16)
    return dict(hidden=_pad_columns(hidden, _pitch(d, "bf16")), weight=weight,
                logits=torch.zeros(T, _pitch(V, case["dtype"]), dtype=_type(case), device=DEV))


def _prepare_clip(case, gen):
    grads = []
    for i, shape in enumerate(_gradient_shapes(case)):
        g = torch.randn(shape, generator=gen, device=DEV).mul_(0.002 * (1 + i % 5))
        grads.append(g.to(_type(case)))
    total = sum(g.numel() * (0.002 * (1 + i % 5)) ** 2 for i, g in enumerate(grads)) ** 0.5
    # (kept apart from the gradients, so that a second pass finds the same ones)
    return dict(grads=grads, outs=[torch.empty_like(g) for g in grads], max_norm=0.37 * total,
                sum_sq=torch.empty(1, dtype=torch.float64, device=DEV), norm=torch.empty(1, device=DEV),
                coef=torch.empty(1, device=DEV))


# ---- one pass ---------------------------------------------------------------------------------------------------


def run(s):
    if own:
        return {"verify": _own_verify, "quantize": _own_quantize, "logits": _own_logits, "clip": _own_clip}[s["case"]["op"]](s)
    return {"verify": _plain_verify, "quantize": _plain_quantize, "logits": _plain_logits, "clip": _plain_clip}[s["case"]["op"]](s)


def _log_softmax(s):
    m = s.amax(dim=-1, keepdim=True)
    return s - m - (s - m).exp().sum(dim=-1, keepdim=True).log()


def _first_max(x):
    at = torch.arange(x.shape[-1], device=x.device).expand_as(x)
    return torch.where(x == x.amax(dim=-1, keepdim=True), at, x.shape[-1]).amin(dim=-1)


def _plain_verify(s):
    """In 64 bits: whether a token is accepted hangs on borders."""
    case = s["case"]
    B, K, V = case["B"], case["K"], case["V"]
    tau = s["temperature"].double()
    greedy = tau == 0
    tau = torch.where(greedy, torch.ones_like(tau), tau)
    place = torch.arange(K + 1, device=DEV)
    lens = s["draft_lens"].long()
    ids = s["draft_ids"].view(B, K + 1).long()
    z = s["target"][:, :V].view(B, K + 1, V)
    logp = _log_softmax(z.double() / tau[:, None, None])
    p_x = logp.gather(2, ids[:, :, None])[:, :, 0].exp()
    if case["draft"]:
        logq = _log_softmax(s["draft"][:, :V].view(B, K + 1, V).double() / tau[:, None, None])
        q_x = logq.gather(2, ids[:, :, None])[:, :, 0].exp()
    else:
        q_x = torch.ones_like(p_x)
    passes = torch.where(greedy[:, None], ids == _first_max(z), s["accept_u"].view(B, K + 1).double() * q_x < p_x)
    n = (passes & (place < lens[:, None])).long().cumprod(dim=1).sum(dim=1)
    sample = torch.arange(B, device=DEV)
    p = logp[sample, n].exp()
    if case["draft"]:
        q = logq[sample, n].exp()
    else:
        q = torch.zeros_like(p).scatter_(1, ids[sample, n][:, None], 1.0)
    left = torch.where((n < lens)[:, None], (p - q).clamp(min=0.0), p)
    left = torch.where((left > 0).any(dim=1, keepdim=True), left, p)
    token = torch.where(greedy, _first_max(z[sample, n]), _first_max(left / s["noise"][:, :V].double()))
    out = torch.where(place == n[:, None], token[:, None], ids)
    mask = place <= n[:, None]
    out_logp = torch.where(mask, logp.gather(2, out[:, :, None])[:, :, 0], 0.0)
    return dict(n_accepted=n.int(), out_ids=torch.where(mask, out, -1).int().view(-1), out_logp=out_logp.float().view(-1),
                out_mask=mask.to(torch.uint8).view(-1))


def _to_blocks(x):
    """The values that x holds in 4-bit blocks: 32 entries share a power of two, each one of 0, .5, 1, 1.5, 2, 3, 4, 6."""
    R, d = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -d % 32)).view(R, -1, 32)
    top = b.abs().amax(dim=2, keepdim=True)
    shared = torch.exp2((torch.frexp(top)[1] - 3).clamp(min=-126).float())         # top = m 2^e, m in [1/2, 1)
    a = b / shared
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    return ((a / step).round() * step).clamp(-6.0, 6.0).mul(shared).view(R, -1)[:, :d]


def _plain_quantize(s):
    return _pad_columns(_to_blocks(s["x"][:, :s["case"]["d"]]).to(torch.bfloat16), s["values"].shape[1])


def _plain_logits(s):
    case = s["case"]
    d = case["d"]
    z = _to_blocks(s["hidden"][:, :d]) @ s["weight"][:, :d].float().t()
    return _pad_columns(z.to(_type(case)), s["logits"].shape[1])


def _plain_clip(s):
    grads = [g.float() for g in s["grads"]]
    sum_sq = torch.stack([g.square().sum(dtype=torch.float64) for g in grads]).sum()
    norm = sum_sq.sqrt()
    coef = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    return dict(norm=norm.float().view(1), coef=coef.float().view(1),
                outs=[(g * coef.float()).to(s["grads"][0].dtype) for g in grads])


# ---- the same with this library ---------------------------------------------------------------------------------


def _workspace(nbytes):
    """A workspace, which a program keeps from call to call."""
    from paper_2605_17862_amd import binding as fb
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=DEV)
    off = (-ws.data_ptr()) % 256
    ws = ws[off:off + nbytes]
    fb.fopd_workspace_init(ws)
    return ws


def _dt(t):
    from paper_2605_17862_amd import binding as fb
    return fb.FOPD_F32 if t.dtype == torch.float32 else fb.FOPD_BF16


def _own_verify(s):
    from paper_2605_17862_amd import binding as fb
    case = s["case"]
    B, K, V = case["B"], case["K"], case["V"]
    R, ld = s["target"].shape
    if "ws" not in s:
        s["ws"] = _workspace(fb.fopd_verify_workspace_bytes(R, V, B))
    fb.fopd_verify_draft(s["target"], s["draft"], _dt(s["target"]), R, V, ld, ld, s["draft_ids"], None, s["draft_lens"], B, K,
                         s["temperature"], s["accept_u"], s["noise"], ld, s["n_accepted"], s["out_ids"], s["out_logp"],
                         s["out_mask"], s["ws"])
    return {k: s[k] for k in ("n_accepted", "out_ids", "out_logp", "out_mask")}


def _own_quantize(s):
    from paper_2605_17862_amd import binding as fb
    R, d = s["case"]["R"], s["case"]["d"]
    if "packed" not in s:
        s["packed"] = torch.empty(fb.fopd_mx4_bytes(R, d), dtype=torch.uint8, device=DEV)
    fb.fopd_mx4_quantize(s["x"], _dt(s["x"]), R, d, s["x"].shape[1], s["packed"])
    fb.fopd_mx4_dequantize(s["packed"], R, d, s["values"], fb.FOPD_BF16, s["values"].shape[1])
    return s["values"]


def _own_logits(s):
    from paper_2605_17862_amd import binding as fb
    T, V, d = s["case"]["T"], s["case"]["V"], s["case"]["d"]
    if "packed" not in s:                                            # the projection is laid out once
        s["packed"] = torch.empty(fb.fopd_mx4_bytes(V, d), dtype=torch.uint8, device=DEV)
        fb.fopd_mx4_quantize(s["weight"], fb.FOPD_BF16, V, d, s["weight"].shape[1], s["packed"])
        s["ws"] = _workspace(fb.fopd_mx4_logits_workspace_bytes(T, V, d))
    fb.fopd_mx4_logits(s["hidden"], fb.FOPD_BF16, s["hidden"].shape[1], s["packed"], T, V, d, s["logits"], _dt(s["logits"]),
                       s["logits"].shape[1], s["ws"])
    return s["logits"]


def _own_clip(s):
    from paper_2605_17862_amd import binding as fb
    if "list" not in s:                                              # the addresses and sizes of the gradients
        s["list"] = fb.grad_tensors(s["grads"], s["outs"])
        s["ws"] = _workspace(fb.fopd_grad_workspace_bytes())
    fb.fopd_grad_norm(s["list"], s["sum_sq"], s["norm"], s["ws"])
    fb.fopd_grad_clip(s["list"], s["sum_sq"], s["max_norm"], EPS, s["coef"])
    return dict(norm=s["norm"], coef=s["coef"], outs=s["outs"])


# ---- what a pass cannot do without ------------------------------------------------------------------------------


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "verify":
        # a greedy sample needs neither the drafter's rows nor random numbers
        V, total = case["V"], 0
        for n, greedy in zip(_lens(case), _is_greedy(case)):
            total += (n + 1) * V * e + (0 if greedy else V * 4 + (n * V * e if case["draft"] else 0))
        return {"bytes": total + case["B"] * (case["K"] + 1) * 17, "flops": 0}
    if case["op"] == "quantize":
        n = case["R"] * case["d"]
        return {"bytes": n * e + 2 * n * 17 // 32 + n * 2, "flops": 0}
    if case["op"] == "logits":
        T, V, d = case["T"], case["V"], case["d"]
        return {"bytes": V * d * 17 // 32 + T * d * 2 + T * V * e, "flops": 2 * T * V * d}
    n = sum(math.prod(s) for s in _gradient_shapes(case))
    return {"bytes": 3 * n * e, "flops": 0}


# ---- the definition, in 64 bits ---------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"verify": _exact_verify, "quantize": _exact_quantize, "logits": _exact_logits, "clip": _exact_clip}[case["op"]](case, s)


def _exact_verify(case, s):
    B, K, V = case["B"], case["K"], case["V"]
    taus, ids, u = s["temperature"].tolist(), s["draft_ids"].tolist(), s["accept_u"].double().tolist()
    n_accepted, out_ids, out_logp, out_mask = [], [-1] * len(ids), [0.0] * len(ids), [0] * len(ids)
    for i, length in enumerate(_lens(case)):
        accepted = 0
        while True:
            r = i * (K + 1) + accepted
            z = s["target"][r, :V].double() / (taus[i] or 1.0)
            lp = z - torch.logsumexp(z, 0)
            q = torch.zeros(V, dtype=torch.float64, device=DEV)
            if accepted == length:
                x = None
            else:
                x = ids[r]
                if case["draft"] and taus[i] > 0:
                    q = torch.softmax(s["draft"][r, :V].double() / taus[i], 0)
                else:
                    q[x] = 1.0
                hit = x == int(torch.nonzero(z == z.max())[0, 0]) if taus[i] == 0 else u[r] * float(q[x]) < math.exp(float(lp[x]))
                if hit:
                    out_ids[r], out_logp[r], out_mask[r] = x, float(lp[x]), 1
                    accepted += 1
                    continue
            if taus[i] == 0:
                race = z
            else:
                rest = torch.clamp(torch.exp(lp) - q, min=0.0)
                race = (rest if float(rest.max()) > 0 else torch.exp(lp)) / s["noise"][i, :V].double()
            x = int(torch.nonzero(race == race.max())[0, 0])
            out_ids[r], out_logp[r], out_mask[r] = x, float(lp[x]), 1
            n_accepted.append(accepted)
            break
    return dict(n_accepted=torch.tensor(n_accepted, dtype=torch.int32), out_ids=torch.tensor(out_ids, dtype=torch.int32),
                out_logp=torch.tensor(out_logp, dtype=torch.float64), out_mask=torch.tensor(out_mask, dtype=torch.uint8))


def _exact_blocks(x):
    """Each entry at the nearest of the fifteen values, ties to the one whose place among the eight magnitudes is even."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    out = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[1], 32):
        b = x[:, c:c + 32].double()
        top = b.abs().amax(dim=1, keepdim=True)
        e = torch.floor(torch.log2(top.clamp(min=1e-300)))
        e = torch.where(torch.exp2(e) > top, e - 1, e)
        e = torch.where(torch.exp2(e + 1) <= top, e + 1, e)
        unit = torch.exp2((e - 2).clamp(min=-127))
        a = (b.abs() / unit).clamp(max=6.0)
        hi = torch.searchsorted(grid, a.contiguous()).clamp(max=7)
        lo = (hi - 1).clamp(min=0)
        up, down = grid[hi] - a, a - grid[lo]
        pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
        out[:, c:c + 32] = torch.where(b < 0, -grid[pick], grid[pick]) * unit
    return out


def _exact_quantize(case, s):
    return _pad_columns(_exact_blocks(s["x"][:, :case["d"]]), s["values"].shape[1])


def _exact_logits(case, s):
    z = _exact_blocks(s["hidden"][:, :case["d"]]) @ s["weight"][:, :case["d"]].double().t()
    return _pad_columns(z, s["logits"].shape[1])


def _exact_clip(case, s):
    total = 0.0
    for g in s["grads"]:
        total = total + (g.double() ** 2).sum()
    norm = torch.sqrt(total)
    c = s["max_norm"] / (norm + EPS)
    c = torch.where(c > 1.0, torch.ones_like(c), c)
    return dict(norm=norm.view(1), coef=c.view(1), outs=[g.double() * c for g in s["grads"]])
