"""What the 8-bit heads and the losses on the head's logits are measured on.

An *i8* case is a head whose weights are kept in 8 bits (one scale for each vocabulary row) and whose hidden states are
rounded to 8 bits by the call (one scale for each hidden row): the full vocabulary, or the active rows of several
sequences.  A *logprob* case asks for the log-probabilities of given tokens, over the full vocabulary or over the active
sets.  A *policy* case is a clipped policy loss with a KL term, a *pair* case a preference loss over pairs of answers;
both return the loss, the tokens' log-probabilities and the gradient of the logits.

With `own` false the operators are computed in elementary torch operations, with it true by the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.04       # policy loss
BETA, SMOOTH = 0.1, 0.05                        # preference loss
LARGEST = 1.6e9                                 # bytes that the largest drawn case moves


def listed():
    return [
        # a small model's draft, one user: latency is all there is
        dict(kind="i8", name="i8_small", V=32000, d=512, batch=1, n=347, M=4),
        # one user of an 8B-class model, a narrow draft over some thousand active rows
        dict(kind="i8", name="i8_draft", V=128256, d=4096, batch=1, n=3000, M=8),
        # a wide draft tree on a 7B-class head
        dict(kind="i8", name="i8_tree", V=152064, d=3584, batch=1, n=3000, M=64),
        # many users of one server, each with an active set of its own
        dict(kind="i8", name="i8_batch", V=128256, d=4096, batch=64, n=2300, M=8),
        # the full-vocabulary step
        dict(kind="i8", name="i8_dense_step", V=128256, d=4096, batch=1, n=0, M=8),
        # all positions of a prompt, or of the answers that a reference model scores
        dict(kind="i8", name="i8_prefill", V=128256, d=4096, batch=1, n=0, M=1024),
        # the draft's own probabilities of what it proposed, over the active sets of many users
        dict(kind="logprob", name="logprob_active", V=128256, batch=64, n=2300, rows=512, type="f32"),
        # a reference model's log-probabilities of a few answers
        dict(kind="logprob", name="logprob_dense", V=128256, batch=1, n=0, rows=509, type="f32"),
        # a handful of tokens of a small model: latency
        dict(kind="policy", name="policy_small", V=32000, rows=7, type="f32", grad="f32"),
        # one training step on answers of two thousand tokens
        dict(kind="policy", name="policy_step", V=128256, rows=2048, type="f32", grad="bf16"),
        # one pair of short answers
        dict(kind="pair", name="pair_small", V=32000, rows=37, pairs=1, type="f32", grad="f32"),
        # a batch of pairs on a 7B-class vocabulary, logits kept in 16 bits
        dict(kind="pair", name="pair_step", V=152064, rows=1021, pairs=8, type="bf16", grad="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["i8", "i8", "logprob", "policy", "pair"])
        V = _log(rng, 4001, 152064)
        if kind == "i8":
            d = 16 * _log(rng, 16, 512)
            if rng.random() < 0.5:
                c = dict(kind=kind, V=V, d=d, batch=1, n=0, M=_log(rng, 1, 1024))
            else:
                batch = rng.choice([1, 1, 2, 5, 16, 64])
                c = dict(kind=kind, V=V, d=d, batch=batch, n=min(V // 2, _log(rng, 50, 9000)), M=_log(rng, 1, 64))
        elif kind == "logprob":
            batch = rng.choice([1, 3, 16, 64])
            n = rng.choice([0, min(V // 2, _log(rng, 50, 9000))])
            c = dict(kind=kind, V=V, batch=batch if n else 1, n=n, rows=(batch if n else 1) * _log(rng, 1, 16 if n else 1500), type=rng.choice(["f32", "bf16"]))
        elif kind == "policy":
            c = dict(kind=kind, V=V, rows=_log(rng, 1, 2048), type=rng.choice(["f32", "bf16"]), grad=rng.choice(["f32", "bf16"]))
        else:
            pairs = rng.choice([1, 2, 7, 16])
            c = dict(kind=kind, V=V, rows=pairs * _log(rng, 4, 500), pairs=pairs, type=rng.choice(["f32", "bf16"]), grad=rng.choice(["f32", "bf16"]))
        w = work(c)
        if w["bytes"] <= LARGEST and w["flops"] <= 1.1e12:
            return c


def _counts(case):
    """live rows of each sequence's active set: ragged around the case's number"""
    return [max(1, case["n"] - 13 * (b % 16)) for b in range(case["batch"])]


def _capacity(case):
    return -(-min(1 + case["n"], case["V"]) // 64) * 64


def _distinct(case):
    """how many distinct rows the active sets of all sequences hold, from the distribution they are drawn from"""
    if case["batch"] == 1:
        return case["n"]
    p = 1.0 / np.power(np.arange(1, case["V"] + 1, dtype=np.float64), 1.1)
    absent = np.zeros(case["V"])
    for n in set(_counts(case)):
        lo, hi = 0.0, 1e9
        for _ in range(80):
            mid = (lo + hi) / 2
            lo, hi = (mid, hi) if (1 - np.exp(-mid * p)).sum() < n else (lo, mid)
        absent -= lo * p * sum(c == n for c in _counts(case))
    return float((1 - np.exp(absent)).sum())


def work(case):
    V, size = case["V"], {"f32": 4, "bf16": 2}
    if case["kind"] == "i8":
        d, rows = case["d"], case["batch"] * case["M"]
        live = sum(_counts(case)) if case["n"] else V
        read = (_distinct(case) if case["n"] else V) * (d + 4)
        return {"bytes": read + 2 * rows * d + 4 * case["M"] * live, "flops": 2 * case["M"] * live * d}
    z = size[case["type"]]
    if case["kind"] == "logprob":
        live = sum(_counts(case)) * (case["rows"] // case["batch"]) if case["n"] else case["rows"] * V
        return {"bytes": live * z + 8 * case["rows"], "flops": 4 * live}
    return {"bytes": case["rows"] * (V * (z + size[case["grad"]]) + 28), "flops": 8 * case["rows"] * V}


def _active(case, g):
    """ascending active ids of every sequence, drawn from a Zipf distribution over a permuted vocabulary"""
    V, counts, cap = case["V"], _counts(case), _capacity(case)
    p = torch.pow(torch.arange(1, V + 1, device="cuda", dtype=torch.float32), -1.1)[torch.randperm(V, device="cuda", generator=g)]
    key = p / torch.empty((case["batch"], V), device="cuda").exponential_(generator=g)
    best = key.topk(max(counts), dim=1).indices
    n = torch.tensor(counts, device="cuda", dtype=torch.int32)
    place = torch.arange(max(counts), device="cuda")
    ids = torch.where(place < n[:, None], best, V).sort(dim=1).values
    out = torch.zeros((case["batch"], cap), dtype=torch.int32, device="cuda")
    out[:, : max(counts)] = torch.where(ids < V, ids, 0)
    return out, n


def _state(case, s, d, M):
    """the library's state with the active sets"""
    from paper_2605_26444_amd import binding as B

    counts, off = _counts(case), np.zeros(case["batch"] + 1, np.int32)
    off[1:] = np.cumsum(counts)
    flat = torch.cat([s["ids"][b, :n] for b, n in enumerate(counts)])
    st = B.State(case["V"], d, case["batch"], 1, max(counts), M, 1)
    B.nanospec_vocab_init(st.h, None, np.zeros(case["batch"] + 1, np.int32), flat, off)
    assert st.capacity == _capacity(case)
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["n" if "n" in case else "rows"] and case["kind"] in ("i8", "logprob") and case["n"]:
        s["ids"], s["n"] = _active(case, g)
    return (_prepare_head if case["kind"] == "i8" else _prepare_rows)(case, s, g)


def _quantized(x):
    """rows in 8 bits and their scales: q = round(127 x / max|x|), scale = max|x| / 127"""
    x = x.float()
    top = x.abs().amax(dim=-1, keepdim=True)
    q = torch.where(top > 0, torch.round(x * 127 / top), torch.zeros_like(x))
    return q, top / 127


def _prepare_head(case, s, g):
    V, d, batch, M = case["V"], case["d"], case["batch"], case["M"]
    s["W"], s["Ws"] = torch.empty((V, d), dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    for v in range(0, V, 16384):
        w = torch.empty((min(16384, V - v), d), device="cuda").normal_(0, 0.02, generator=g).bfloat16()
        q, t = _quantized(w)
        s["W"][v : v + 16384], s["Ws"][v : v + 16384] = q.to(torch.int8), t[:, 0]
    shape = (batch, M, d) if case["n"] else (M, d)
    s["H"] = torch.empty(shape, device="cuda").normal_(generator=g).bfloat16()
    s["out"] = torch.zeros((batch, M, _capacity(case)) if case["n"] else (M, V), device="cuda")
    if own:
        from paper_2605_26444_amd import binding as B

        s["bytes"] = B.nanospec_head_i8_workspace(batch * M, d)
        s["ws"] = torch.empty(s["bytes"], dtype=torch.uint8, device="cuda")
        if case["n"]:
            s["st"] = _state(case, s, d, M)
    return s


def _prepare_rows(case, s, g):
    V, rows = case["V"], case["rows"]
    listed_rows = "ids" in s
    width = _capacity(case) if listed_rows else V
    z = torch.empty((rows, width), device="cuda").normal_(0, 2, generator=g)
    if listed_rows:
        each = rows // case["batch"]
        live = s["n"].repeat_interleave(each)
        col = (torch.rand(rows, device="cuda", generator=g) * live).long()
        s["tokens"] = s["ids"].repeat_interleave(each, 0).gather(1, col[:, None])[:, 0].contiguous()
    else:
        col = torch.randint(0, V, (rows,), device="cuda", generator=g)
        s["tokens"] = col.to(torch.int32)
    # tokens that a policy has chosen are likely ones
    z.scatter_add_(1, col[:, None], torch.empty((rows, 1), device="cuda").normal_(7, 3, generator=g))
    s["z"] = z.to(_TYPE[case["type"]])
    s["logprob"] = torch.zeros(rows, device="cuda")
    if case["kind"] != "logprob":
        lp = _stats(s["z"], col)[0].float()
        normal = lambda sigma: torch.empty(rows, device="cuda").normal_(0, sigma, generator=g)
        s["old"], s["ref"] = lp + normal(0.15), lp + normal(0.4)
        answer = (torch.rand(rows, device="cuda", generator=g) > 0.1).float()          # the others are prompt or padding
        s["grad"] = torch.zeros((rows, V), dtype=_TYPE[case["grad"]], device="cuda")
        s["loss"] = torch.zeros(1, device="cuda")
        if case["kind"] == "policy":
            s["adv"] = normal(1.0)
            s["weight"] = answer / answer.sum().clamp(min=1)
            s["row_loss"] = torch.zeros(rows, device="cuda")
        else:
            s["weight"] = answer
            s["off"] = _offsets(case)
            s["margin"] = torch.zeros(case["pairs"], device="cuda")
    if own:
        from paper_2605_26444_amd import binding as B

        if listed_rows:
            s["st"] = _state(case, s, 16, 1)
            s["rows"] = B.logit_rows(s["z"], s["tokens"], V=width, ids=s["st"].ids_ptr, n=s["st"].n_ptr, rows_per_list=rows // case["batch"])
        else:
            s["rows"] = B.logit_rows(s["z"], s["tokens"])
        s["bytes"] = B.nanospec_loss_workspace(rows, width)
        s["ws"] = torch.empty(s["bytes"], dtype=torch.uint8, device="cuda")
    return s


_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _offsets(case):
    """first row of every answer, chosen and rejected in turn, of uneven lengths, the last rows padding"""
    seqs, rows = 2 * case["pairs"], case["rows"] - case["rows"] // 32
    cut = [rows * i // seqs + ((i * 5) % 7 - 3) * (rows // seqs) // 8 for i in range(seqs)]
    return np.array([0] + cut[1:] + [rows], np.int32)


def run(state):
    if own:
        return _RUN_OWN[state["case"]["kind"]](state)
    return _RUN_PLAIN[state["case"]["kind"]](state)


# ---- the library -------------------------------------------------------------------------------------------------


def _own_i8(s):
    from paper_2605_26444_amd import binding as B

    c = s["case"]
    if c["n"]:
        B.nanospec_sparse_head_i8(s["st"].h, s["W"], s["Ws"], s["H"], c["M"], s["out"], s["ws"], s["bytes"])
    else:
        B.nanospec_dense_head_i8(s["W"], s["Ws"], s["H"], c["V"], c["d"], c["M"], s["out"], s["ws"], s["bytes"])
    return s["out"]


def _own_logprob(s):
    from paper_2605_26444_amd import binding as B

    B.nanospec_token_logprob(s["rows"], s["logprob"], s["ws"], s["bytes"])
    return s["logprob"]


def _own_policy(s):
    from paper_2605_26444_amd import binding as B

    B.nanospec_policy_loss(s["rows"], s["old"], s["ref"], s["adv"], s["weight"], CLIP_LOW, CLIP_HIGH, KL, s["loss"], s["row_loss"], s["logprob"],
                           s["grad"], s["ws"], s["bytes"])
    return {"loss": s["loss"], "row_loss": s["row_loss"], "logprob": s["logprob"], "grad": s["grad"]}


def _own_pair(s):
    from paper_2605_26444_amd import binding as B

    B.nanospec_preference_loss(s["rows"], s["off"], s["ref"], s["weight"], BETA, SMOOTH, s["loss"], s["margin"], s["logprob"], s["grad"],
                               s["ws"], s["bytes"])
    return {"loss": s["loss"], "margin": s["margin"], "logprob": s["logprob"], "grad": s["grad"]}


_RUN_OWN = {"i8": _own_i8, "logprob": _own_logprob, "policy": _own_policy, "pair": _own_pair}


# ---- the plain forms ---------------------------------------------------------------------------------------------


def _live(s, width):
    return torch.arange(width, device="cuda") < s["n"][:, None]


def _plain_i8(s):
    c = s["case"]
    q, t = _quantized(s["H"])
    if not c["n"]:
        return torch.matmul(q, s["W"].float().t()) * t * s["Ws"]
    rows = s["W"][s["ids"].long()].float()                                # [batch][capacity][d]
    z = torch.matmul(q, rows.transpose(1, 2).contiguous()) * t * s["Ws"][s["ids"].long()][:, None]
    return torch.where(_live(s, z.shape[2])[:, None], z, torch.zeros_like(z))


def _stats(z, col):
    """log-probability of the columns in 64 bits, and each row's probabilities, from sums in 32"""
    z = z.float()
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lp = (z.gather(1, col.long()[:, None]) - top).double() - torch.log(total.double())
    return lp[:, 0], e, total


def _plain_logprob(s):
    c, z = s["case"], s["z"]
    col = s["tokens"]
    if c["n"]:
        each = c["rows"] // c["batch"]
        z = torch.where(_live(s, z.shape[1]).repeat_interleave(each, 0), z.float(), torch.full_like(z, -math.inf, dtype=torch.float32))
        ids = torch.where(_live(s, z.shape[1]), s["ids"], c["V"])
        col = torch.searchsorted(ids, s["tokens"].view(c["batch"], each).contiguous()).view(-1)
    return _stats(z, col)[0].float()


def _gradient(s, e, total, dlp):
    """dlp * (the token's indicator - probabilities)"""
    dlp = dlp.float()[:, None]
    g = e * (-dlp / total)
    g.scatter_add_(1, s["tokens"].long()[:, None], dlp)
    return g.to(_TYPE[s["case"]["grad"]])


def _plain_policy(s):
    lp, e, total = _stats(s["z"], s["tokens"])
    row, dlp, loss = _policy(lp, s)
    return {"loss": loss.float(), "row_loss": row.float(), "logprob": torch.where(s["weight"] != 0, lp, 0).float(), "grad": _gradient(s, e, total, dlp)}


def _policy(lp, s):
    """rows' losses, derivatives by the log-probability and the weighted sum, in lp's type"""
    old, ref, adv, w = (s[k].to(lp.dtype) for k in ("old", "ref", "adv", "weight"))
    ratio, gap = torch.exp(lp - old), ref - lp
    free, held = ratio * adv, torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv
    row = -torch.minimum(free, held) + KL * (torch.exp(gap) - gap - 1)
    row = torch.where(w != 0, row, torch.zeros_like(row))
    dlp = w * (torch.where(free <= held, -free, torch.zeros_like(free)) + KL * (1 - torch.exp(gap)))
    return row, dlp, (w * row).sum().reshape(1)


def _plain_pair(s):
    lp, e, total = _stats(s["z"], s["tokens"])
    margin, dlp, loss, counted = _pair(lp, s)
    return {"loss": loss.float(), "margin": margin.float(), "logprob": torch.where(counted, lp, 0).float(), "grad": _gradient(s, e, total, dlp)}


def _pair(lp, s):
    """margins of the pairs, derivatives by the log-probability, the mean loss and the rows that count, in lp's type"""
    pairs = s["case"]["pairs"]
    off = torch.from_numpy(s["off"].astype(np.int64)).cuda()
    place = torch.arange(len(lp), device="cuda")
    seq = torch.searchsorted(off, place, right=True) - 1                  # 2 pairs: behind the last answer
    inside = seq < 2 * pairs
    w = torch.where(inside, s["weight"], 0).to(lp.dtype)
    ratio = torch.where(w != 0, w * (lp - s["ref"].to(lp.dtype)), 0)
    upto = torch.cat([torch.zeros(1, dtype=lp.dtype, device="cuda"), torch.cumsum(ratio, 0)])
    sums = upto[off[1:]] - upto[off[:-1]]
    margin = BETA * (sums[0::2] - sums[1::2])
    loss = ((1 - SMOOTH) * torch.log1p(torch.exp(-margin)) + SMOOTH * torch.log1p(torch.exp(margin))).mean().reshape(1)
    dm = -(1 - SMOOTH) / (1 + torch.exp(margin)) + SMOOTH / (1 + torch.exp(-margin))
    sign = 1.0 - 2.0 * (seq % 2).to(lp.dtype)
    dlp = torch.where(inside, sign * BETA / pairs * dm[torch.clamp(seq // 2, max=pairs - 1)] * w, 0)
    return margin, dlp, loss, w != 0


_RUN_PLAIN = {"i8": _plain_i8, "logprob": _plain_logprob, "policy": _plain_policy, "pair": _plain_pair}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "i8":
        return _exact_head(s)
    z = s["z"].double()
    col = s["tokens"].long()
    if case["kind"] == "logprob" and case["n"]:
        each = case["rows"] // case["batch"]
        owner = torch.arange(case["rows"], device="cuda") // each
        z = z.masked_fill(torch.arange(z.shape[1], device="cuda") >= s["n"][owner][:, None], -math.inf)
        same = (s["ids"][owner] == s["tokens"][:, None]) & (torch.arange(z.shape[1], device="cuda") < s["n"][owner][:, None])
        col = same.to(torch.int8).argmax(dim=1)
    lp_all = z - torch.logsumexp(z, dim=1, keepdim=True)
    lp = lp_all[torch.arange(case["rows"], device="cuda"), col]
    if case["kind"] == "logprob":
        return lp
    lp = lp.requires_grad_(True)
    w = s["weight"].double()
    if case["kind"] == "policy":
        ratio = torch.exp(lp - s["old"].double())
        a = s["adv"].double()
        gap = s["ref"].double() - lp
        row = torch.maximum(-ratio * a, -torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * a) + KL * (torch.expm1(gap) - gap)
        loss = (w * row).sum()
        counted, more = w != 0, {"row_loss": torch.where(w != 0, row, 0).detach()}
    else:
        off, terms = s["off"], []
        counted = torch.zeros(case["rows"], dtype=torch.bool, device="cuda")
        for p in range(case["pairs"]):
            total = lp.new_zeros(())
            for sign, q in ((1, 2 * p), (-1, 2 * p + 1)):
                part = slice(int(off[q]), int(off[q + 1]))
                total = total + sign * (w[part] * (lp[part] - s["ref"][part].double())).sum()
                counted[part] = w[part] != 0
            terms.append(BETA * total)
        margin = torch.stack(terms)
        good, bad = -torch.nn.functional.softplus(-margin), -torch.nn.functional.softplus(margin)
        loss = -((1 - SMOOTH) * good + SMOOTH * bad).mean()
        more = {"margin": margin.detach()}
    (dlp,) = torch.autograd.grad(loss, lp)
    grad = -dlp[:, None] * torch.exp(lp_all)
    grad[torch.arange(case["rows"], device="cuda"), col] += dlp
    return {"loss": loss.detach().reshape(1), "logprob": torch.where(counted, lp, 0).detach(), "grad": grad, **more}


def _exact_head(s):
    c = s["case"]
    h = s["H"].double()
    top = h.abs().amax(dim=-1, keepdim=True)
    q = torch.round(h * 127 / top) * (top / 127)
    if not c["n"]:
        out = torch.empty((c["M"], c["V"]), dtype=torch.float64, device="cuda")
        for v in range(0, c["V"], 32768):
            out[:, v : v + 32768] = q @ (s["W"][v : v + 32768].double() * s["Ws"][v : v + 32768].double()[:, None]).t()
        return out
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_counts(c)):
        ids = s["ids"][b, :n].long()
        out[b, :, :n] = q[b] @ (s["W"][ids].double() * s["Ws"][ids].double()[:, None]).t()
    return out
