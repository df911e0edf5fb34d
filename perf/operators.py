"""Operators of workers that fine-tune a large shared model, as timed cases.

Every worker trains low-rank adapters beside a frozen projection that all share; the adapters are its row of the parameter
matrix, so the consensus mix runs over them.  The losses are over a vocabulary.  `op` names the call:

  forward    the projection with the workers' adapters: training batches, and serving with a row or a few per worker
  backward   gradients of the adapters (rows of the gradient matrix) and of the projection's input
  distill    loss and gradient of distillation from a teacher's top logits
  policy     loss and gradient of the clipped policy objective with a KL term
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}
SCALE = 2.0          # alpha / rank of the adapters
CLIP = (0.2, 0.28)   # the policy ratio stays in [1 - CLIP[0], 1 + CLIP[1]]
KL = 0.04


# ------------------------------------------------------------------------------------------ the cases
def _projection(op, workers, rows, inp, out, rank, spread, bias=False):
    return dict(op=op, workers=workers, rows=rows, inp=inp, out=out, rank=rank, spread=spread, bias=bias)


def _distill(workers, rows, vocab, top, dtype, tau, masked):
    return dict(op="distill", workers=workers, rows=rows, vocab=vocab, top=top, dtype=dtype, tau=tau, masked=masked)


def _policy(workers, rows, vocab, dtype, tau, masked, reference=True):
    return dict(op="policy", workers=workers, rows=rows, vocab=vocab, dtype=dtype, tau=tau, masked=masked, reference=reference)


def listed():
    return [
        # Serving: a decoding step, one row for each of a few workers; latency, and the bytes of the weights.
        dict(_projection("forward", 8, 8, 1024, 1024, 16, "even"), name="decode_8"),
        # A decoding step of more requests on a wider layer; some workers have several requests, some none.
        dict(_projection("forward", 64, 100, 4096, 4096, 16, "ragged"), name="decode_100"),
        # A training batch of ragged sequences on odd sizes, with a bias.
        dict(_projection("forward", 24, 1999, 1000, 1336, 12, "ragged", bias=True), name="forward_ragged"),
        # The largest forward pass: eight workers, a thousand tokens each.
        dict(_projection("forward", 8, 8192, 4096, 4096, 16, "even"), name="forward_large"),
        # Gradients of a small training batch, ...
        dict(_projection("backward", 24, 1999, 1000, 1336, 12, "ragged"), name="backward_ragged"),
        # ... and of the largest, at a large rank.
        dict(_projection("backward", 8, 8192, 4096, 4096, 64, "ragged"), name="backward_large"),
        # Distillation: a small vocabulary in fp32 with few rows, ...
        dict(_distill(8, 256, 4096, 16, "fp32", 2.0, 0.0), name="distill_small"),
        # ... an odd one whose rows are not aligned, with prompt tokens that carry no weight, ...
        dict(_distill(16, 2048, 50001, 32, "bf16", 1.0, 0.25), name="distill_odd"),
        # ... and a large one.
        dict(_distill(8, 4096, 131072, 64, "bf16", 2.0, 0.0), name="distill_large"),
        # Policy loss: few tokens of a small vocabulary, ...
        dict(_policy(4, 100, 8191, "fp32", 1.0, 0.0), name="policy_small"),
        # ... fp16 logits, prompts masked, no reference model, ...
        dict(_policy(16, 2000, 32000, "fp16", 0.8, 0.4, reference=False), name="policy_masked"),
        # ... and the largest.
        dict(_policy(8, 4096, 128000, "bf16", 1.0, 0.0), name="policy_large"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "distill", "policy"])
    workers = _log(rng, 1, 64)
    if op in ("forward", "backward"):
        serving = op == "forward" and rng.random() < 0.4
        rows = _log(rng, 1, 128) if serving else _log(rng, 64, 8192)
        inp, out, rank = 8 * _log(rng, 16, 512), 8 * _log(rng, 16, 512), rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 64)])
        return _projection(op, workers, rows, inp, out, rank, rng.choice(["even", "ragged", "ragged"]), rng.random() < 0.3 and op == "forward")
    vocab = _log(rng, 256, 131072)
    rows = _log(rng, 8, min(16384, (1 << 29) // vocab))
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if dtype == "fp32":
        rows = max(8, rows // 2)
    tau, masked = rng.choice([0.7, 1.0, 1.0, 2.0]), rng.choice([0.0, 0.0, 0.25, 0.5])
    if op == "distill":
        return _distill(workers, rows, vocab, rng.choice([1, 8, 16, 32, 64, rng.randint(1, 64)]), dtype, tau, masked)
    return _policy(workers, rows, vocab, dtype, tau, masked, rng.random() < 0.7)


# ------------------------------------------------------------------------------------------ inputs
def _rowstart(case, seed):
    """Where each worker's rows begin: even shares, or cuts at random places (a worker may have none)."""
    n, rows = case["workers"], case["rows"]
    if case.get("spread", "ragged") == "even":
        cuts = [(rows * w) // n for w in range(n + 1)]
    else:
        rng = random.Random(seed)
        cuts = [0] + sorted(rng.randint(0, rows) for _ in range(n - 1)) + [rows]
    return torch.tensor(cuts, dtype=torch.int32, device="cuda")


def _offsets(case):
    """Where a row of the parameter matrix holds the two factors, and its length: blocks start at multiples of 32 floats."""
    up = lambda v: (v + 31) // 32 * 32  # noqa: E731
    b_off = up(case["rank"] * case["inp"])
    return 0, b_off, b_off + up(case["rank"] * case["out"])


def _graph(n):
    """The communication graph that a handle is made for: a ring."""
    if n == 1:
        return np.zeros(2, np.int32), np.zeros(0, np.int32)
    nbrs = [sorted({(i - 1) % n, (i + 1) % n}) for i in range(n)]
    return np.cumsum([0] + [len(v) for v in nbrs]).astype(np.int32), np.concatenate(nbrs).astype(np.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)  # noqa: E731
    n, rows = case["workers"], case["rows"]
    st = {"case": case, "rowstart": _rowstart(case, seed)}
    if case["op"] in ("forward", "backward"):
        k, m, r = case["inp"], case["out"], case["rank"]
        a_off, b_off, ld = _offsets(case)
        X = torch.zeros(n, ld, device="cuda")
        X[:, a_off: a_off + r * k] = normal(n, r * k) / math.sqrt(k)
        X[:, b_off: b_off + r * m] = normal(n, r * m) * (0.25 / math.sqrt(r))
        st.update(X=X, W=(normal(m, k) / math.sqrt(k)).bfloat16(), x=normal(rows, k).bfloat16(), bias=normal(m) if case["bias"] else None)
        if case["op"] == "forward":
            st.update(y=torch.empty(rows, m, dtype=torch.bfloat16, device="cuda"), hidden=torch.empty(rows, r, device="cuda"))
        else:
            worker = torch.bucketize(torch.arange(rows, device="cuda"), st["rowstart"][1:].long(), right=True)
            A = X[:, a_off: a_off + r * k].view(n, r, k)
            hidden = torch.einsum("tk,wrk->twr", st["x"].float(), A)[torch.arange(rows, device="cuda"), worker]
            st.update(hidden=hidden.contiguous(), dy=normal(rows, m).mul_(1e-3).bfloat16(), G=torch.zeros_like(X),
                      d_hidden=torch.empty(rows, r, device="cuda"), dx=torch.empty_like(st["x"]))
    else:
        v, t = case["vocab"], TYPES[case["dtype"]]
        z = torch.empty(rows, v, dtype=t, device="cuda")
        for a in range(0, rows, 512):  # a spread of three, as trained models have: a few tokens carry most of the mass
            z[a: a + 512] = (3.0 * normal(min(512, rows - a), v)).to(t)
        weight = None
        if case["masked"]:
            weight = (torch.rand(rows, device="cuda", generator=gen) >= case["masked"]).float() / max(1.0, rows / n)
        st.update(z=z, dz=torch.empty_like(z), weight=weight, row_loss=torch.empty(rows, device="cuda"), loss=torch.empty(n, device="cuda"))
        if case["op"] == "distill":
            # the teacher agrees with the student on part of its list; a list may end early
            top = case["top"]
            idx = torch.rand(rows, top, device="cuda", generator=gen).mul_((v - top) / top).add_(torch.arange(top, device="cuda") * ((v - top) / top)).long()
            short = torch.rand(rows, device="cuda", generator=gen) < 0.1
            length = torch.where(short, (torch.rand(rows, device="cuda", generator=gen) * top).long() + 1, torch.full((rows,), top, device="cuda"))
            t_logit = 2.0 * normal(rows, top) + 0.5 * z.gather(1, idx).float()
            idx[torch.arange(top, device="cuda")[None] >= length[:, None]] = -1
            st.update(top_idx=idx.int(), top_logit=t_logit)
        else:
            # tokens were sampled from nearly this policy: its own log-probability, a step of an optimiser earlier
            tau = case["tau"]
            action, logp = [], []
            for a in range(0, rows, 512):
                lp = torch.log_softmax(z[a: a + 512].double() / tau, dim=1)
                u = torch.rand(lp.shape, device="cuda", generator=gen, dtype=torch.float64).clamp_(1e-300)
                pick = (lp - (-u.log()).log()).argmax(dim=1)
                action.append(pick)
                logp.append(lp.gather(1, pick[:, None])[:, 0])
            step = 0.2 * normal(rows).double()
            for border in (1.0 - CLIP[0], 1.0 + CLIP[1]):  # on which side of the border a ratio lies is not left to the last bit
                step = torch.where((step.exp() - border).abs() < 1e-4, step + 1e-3, step)
            logp = torch.cat(logp)
            st.update(action=torch.cat(action).int(), old_logp=(logp - step).float(), ref_logp=(logp + 0.3 * normal(rows)).float() if case["reference"] else None,
                      advantage=normal(rows), logp=torch.empty(rows, device="cuda"))
    if own:
        import paper_2102_06280_b200 as dbw
        rowptr, col = _graph(n)
        if case["op"] in ("forward", "backward"):
            layout = dbw.lowrank_layout([(case["inp"], case["out"], case["rank"])])
            st["adapter"], d = layout.adapters[0], layout.ld
        else:
            d = 4
        st["h"] = dbw.Dbw(rowptr, col, d=d, device=torch.cuda.current_device())
    return st


# ------------------------------------------------------------------------------------------ one pass
def _own(st):
    case, h = st["case"], st["h"]
    if case["op"] == "forward":
        h.lowrank_forward(st["adapter"], st["X"], st["W"], st["x"], st["rowstart"], st["y"], st["hidden"], scale=SCALE, bias=st["bias"])
        return {"y": st["y"], "hidden": st["hidden"]}
    if case["op"] == "backward":
        h.lowrank_backward(st["adapter"], st["X"], st["W"], st["x"], st["hidden"], st["dy"], st["rowstart"], st["G"], st["d_hidden"], d_in=st["dx"], scale=SCALE)
        return {"G": st["G"], "d_hidden": st["d_hidden"], "dx": st["dx"]}
    if case["op"] == "distill":
        h.distill(st["z"], st["top_idx"], st["top_logit"], st["rowstart"], st["row_loss"], loss=st["loss"], d_logits=st["dz"], temperature=case["tau"],
                  row_weight=st["weight"])
        return {"row_loss": st["row_loss"], "loss": st["loss"], "dz": st["dz"]}
    h.policy_loss(st["z"], st["action"], st["old_logp"], st["advantage"], st["rowstart"], st["row_loss"], loss=st["loss"], logp=st["logp"], d_logits=st["dz"],
                  ref_logp=st["ref_logp"], temperature=case["tau"], clip_low=CLIP[0], clip_high=CLIP[1], kl_coef=KL if case["reference"] else 0.0,
                  row_weight=st["weight"])
    return {"row_loss": st["row_loss"], "loss": st["loss"], "logp": st["logp"], "dz": st["dz"]}


def _workers_of(st):
    """[rows][workers]: 1 where the row is the worker's."""
    n, rows = st["case"]["workers"], st["case"]["rows"]
    worker = torch.bucketize(torch.arange(rows, device="cuda"), st["rowstart"][1:].long(), right=True)
    return (worker[:, None] == torch.arange(n, device="cuda")).float()


def _factors(st):
    case = st["case"]
    n, k, m, r = case["workers"], case["inp"], case["out"], case["rank"]
    a_off, b_off, _ = _offsets(case)
    return st["X"][:, a_off: a_off + r * k].reshape(n * r, k), st["X"][:, b_off: b_off + r * m].reshape(n * r, m)


def _plain_projection(st):
    # every row times every worker's factor, and of that what the row's own worker has
    case, mine = st["case"], _workers_of(st)
    n, rows, k, m, r = case["workers"], case["rows"], case["inp"], case["out"], case["rank"]
    A, B = _factors(st)
    x, W = st["x"].float(), st["W"].float()
    if case["op"] == "forward":
        h = (x @ A.t()).view(rows, n, r) * mine[:, :, None]
        y = x @ W.t() + SCALE * (h.view(rows, n * r) @ B)
        if st["bias"] is not None:
            y = y + st["bias"]
        return {"y": y.bfloat16(), "hidden": h.sum(dim=1)}
    dy = st["dy"].float()
    u = SCALE * (dy @ B.t()).view(rows, n, r) * mine[:, :, None]
    h = st["hidden"][:, None, :] * mine[:, :, None]
    a_off, b_off, _ = _offsets(case)
    G = torch.zeros_like(st["X"])
    G[:, a_off: a_off + r * k] = (u.view(rows, n * r).t() @ x).view(n, r * k)
    G[:, b_off: b_off + r * m] = SCALE * (h.view(rows, n * r).t() @ dy).view(n, r * m)
    dx = dy @ W + u.view(rows, n * r) @ A
    return {"G": G, "d_hidden": u.sum(dim=1), "dx": dx.bfloat16()}


def _row_weight(st, mine):
    return st["weight"] if st["weight"] is not None else mine @ (1.0 / mine.sum(dim=0).clamp(min=1.0))


def _plain_distill(st):
    case, mine = st["case"], _workers_of(st)
    tau, weight = case["tau"], _row_weight(st, mine)
    z = st["z"].float() / tau
    z = z - z.amax(dim=1, keepdim=True)
    q = z.exp()
    total = q.sum(dim=1, keepdim=True)
    q = q / total
    idx, there = st["top_idx"].long().clamp(min=0), st["top_idx"] >= 0
    t = torch.where(there, st["top_logit"] / tau, -math.inf)
    t = t - t.amax(dim=1, keepdim=True)
    p = t.exp()
    mass = p.sum(dim=1, keepdim=True)
    p = p / mass
    logs = (t - mass.log()) - (z.gather(1, idx) - total.log())
    row = tau * tau * torch.where(there, p * logs, 0.0).sum(dim=1)
    row = torch.where(weight != 0, row, 0.0)
    dz = (q.scatter_add_(1, idx, -p)) * (weight * tau)[:, None]
    return {"row_loss": row, "loss": mine.t() @ (weight * row), "dz": dz.to(st["z"].dtype)}


def _plain_policy(st):
    case, mine = st["case"], _workers_of(st)
    tau, weight, action = case["tau"], _row_weight(st, mine), st["action"].long()[:, None]
    z = st["z"].float() / tau
    z = z - z.amax(dim=1, keepdim=True)
    q = z.exp()
    total = q.sum(dim=1, keepdim=True)
    q = q / total
    logp = (z.gather(1, action) - total.log())[:, 0]
    ratio = (logp - st["old_logp"]).exp()
    adv = st["advantage"]
    free, held = ratio * adv, ratio.clamp(1.0 - CLIP[0], 1.0 + CLIP[1]) * adv
    row, slope = -torch.minimum(free, held), torch.where(free <= held, -free, 0.0)
    if case["reference"]:
        far = st["ref_logp"] - logp
        row, slope = row + KL * (far.exp() - far - 1.0), slope + KL * (1.0 - far.exp())
    row, logp = torch.where(weight != 0, row, 0.0), torch.where(weight != 0, logp, 0.0)
    slope = weight * slope / tau
    dz = (q * -slope[:, None]).scatter_add_(1, action, slope[:, None])
    return {"row_loss": row, "loss": mine.t() @ (weight * row), "logp": logp, "dz": dz.to(st["z"].dtype)}


def run(st):
    if own:
        return _own(st)
    op = st["case"]["op"]
    return _plain_distill(st) if op == "distill" else _plain_policy(st) if op == "policy" else _plain_projection(st)


# ------------------------------------------------------------------------------------------ the definition, in 64 bits
def _exact_projection(case, st):
    cuts = st["rowstart"].tolist()
    a_off, b_off, ld = _offsets(case)
    k, m, r = case["inp"], case["out"], case["rank"]
    x, W = st["x"].double(), st["W"].double()
    y, u, dx = [], [], []
    hidden, G = [], torch.zeros(case["workers"], ld, dtype=torch.float64, device="cuda")
    for w, (a, b) in enumerate(zip(cuts, cuts[1:])):
        A = st["X"][w, a_off: a_off + r * k].double().view(r, k)
        B = st["X"][w, b_off: b_off + r * m].double().view(r, m)
        if case["op"] == "forward":
            hidden.append(torch.einsum("tk,rk->tr", x[a:b], A))
            y.append(torch.einsum("tk,mk->tm", x[a:b], W) + SCALE * hidden[-1] @ B)
        else:
            dy = st["dy"][a:b].double()
            u.append(SCALE * torch.einsum("tm,rm->tr", dy, B))
            G[w, a_off: a_off + r * k] = (u[-1].t() @ x[a:b]).reshape(-1)
            G[w, b_off: b_off + r * m] = SCALE * (st["hidden"][a:b].double().t() @ dy).reshape(-1)
            dx.append(torch.einsum("tm,mk->tk", dy, W) + u[-1] @ A)
    if case["op"] == "forward":
        return {"y": torch.cat(y) + (0.0 if st["bias"] is None else st["bias"].double()), "hidden": torch.cat(hidden)}
    return {"G": G, "d_hidden": torch.cat(u), "dx": torch.cat(dx)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("forward", "backward"):
        return _exact_projection(case, st)
    tau, n, rows = case["tau"], case["workers"], case["rows"]
    sizes = (st["rowstart"][1:] - st["rowstart"][:-1]).long()
    worker = torch.repeat_interleave(torch.arange(n, device="cuda"), sizes)
    weight = st["weight"].double() if st["weight"] is not None else 1.0 / sizes.double()[worker]
    row, logps, dz = [], [], []
    for a in range(0, rows, 256):  # some rows at a time: 64 bits of the largest case do not all fit
        part = slice(a, min(rows, a + 256))
        lq = torch.log_softmax(st["z"][part].double() / tau, dim=1)
        here = torch.arange(lq.shape[0], device="cuda")
        if case["op"] == "distill":
            idx, t = st["top_idx"][part].long(), st["top_logit"][part].double()
            lp = torch.log_softmax(torch.where(idx >= 0, t / tau, torch.full_like(t, -math.inf)), dim=1)
            p = lp.exp()
            target = torch.zeros_like(lq).index_put_((here[:, None].expand_as(idx), idx.clamp(min=0)), p, accumulate=True)
            ls = torch.where(idx >= 0, p * (lp - lq[here[:, None], idx.clamp(min=0)]), torch.zeros_like(t)).sum(dim=1) * tau ** 2
            g = tau * (lq.exp() - target)
        else:
            act, adv = st["action"][part].long(), st["advantage"][part].double()
            logp = lq[here, act]
            logps.append(torch.where(weight[part] != 0, logp, torch.zeros_like(logp)))
            ratio = torch.exp(logp - st["old_logp"][part].double())
            clipped = ((adv > 0) & (ratio > 1 + CLIP[1])) | ((adv < 0) & (ratio < 1 - CLIP[0]))
            bound = torch.where(adv > 0, torch.full_like(adv, 1 + CLIP[1]), torch.full_like(adv, 1 - CLIP[0]))
            ls = -torch.where(clipped, bound, ratio) * adv
            slope = torch.where(clipped, torch.zeros_like(adv), -ratio * adv)
            if case["reference"]:
                ref = torch.exp(st["ref_logp"][part].double() - logp)
                ls = ls + KL * (ref - 1 - torch.log(ref))
                slope = slope + KL * (1 - ref)
            g = -lq.exp() * slope[:, None]
            g[here, act] += slope
            g = g / tau
        live = weight[part] != 0
        row.append(torch.where(live, ls, torch.zeros_like(ls)))
        dz.append((g * weight[part][:, None]).to(torch.float32 if st["z"].dtype != torch.float32 else torch.float64))
    row = torch.cat(row)
    got = {"row_loss": row, "loss": torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, worker, weight * row), "dz": torch.cat(dz)}
    if case["op"] == "policy":
        got["logp"] = torch.cat(logps)
    return got


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    n, rows = case["workers"], case["rows"]
    if case["op"] in ("forward", "backward"):
        k, m, r = case["inp"], case["out"], case["rank"]
        holders = min(n, rows)  # workers that have rows
        if case["op"] == "forward":
            return {"bytes": 2 * (rows * (k + m) + k * m) + 4 * holders * r * (k + m) + 4 * rows * r, "flops": 2 * rows * (k * m + r * (k + m))}
        return {"bytes": 2 * (rows * (2 * k + m) + k * m) + 4 * (holders + n) * r * (k + m) + 8 * rows * r, "flops": 2 * rows * (k * m + 2 * r * (k + m))}
    # logits of the rows that carry weight in, a gradient for every row out
    live = 1.0 - case["masked"]
    size = SIZES[case["dtype"]] * rows * case["vocab"]
    per_row = 8 * case["top"] if case["op"] == "distill" else 20
    return {"bytes": size * (1.0 + live) + rows * (8 + per_row), "flops": 6.0 * rows * live * case["vocab"]}
