"""Losses on logits of every size and on rows at the edges of what they accept, against 64 bits; tolerances are those derived in losses64.py:
a logit's distance from its row's maximum carries one rounding, whatever the maximum is."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import losses64 as L
import test_gpu_losses as T
from paper_2605_26444_amd import binding as B

pytestmark = pytest.mark.gpu


def compare(z, t, old, ref, adv, grad_kind="f32"):
    """log-probabilities, policy loss and preference loss of rows that all count, each with its gradient"""
    rows, V = z.shape
    zd, want = z.cuda(), L.rows64(z.double().numpy(), t)
    out = torch.empty(rows, device="cuda")
    ws, n = T.space(rows, V)
    B.nanospec_token_logprob(B.logit_rows(zd, T.dev(t, torch.int32)), out, ws, n)
    T.near(out.cpu(), T.lp_of(want), T.lp_bound(want), "logprob")
    name = T.NAME[T.KIND[grad_kind]]
    grad = torch.empty((rows, V), dtype=T.KIND[grad_kind], device="cuda")

    def gradients(dlp, slack, what):
        gg = grad.float().cpu().numpy()
        for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 1.0, name)):
            T.near(gg[r], x, b, (what, r))

    got = T.run_policy(zd, t, old, ref, adv, None, 0.05, grad)
    loss, lb, row, rb, dlp, slack = L.policy(want, old, ref, adv, None, 0.2, 0.28, 0.05)
    T.near(got["lp"][:rows], T.lp_of(want), T.lp_bound(want), "policy logprob")
    T.near(got["row"][:rows], row, rb, "rows")
    T.near(got["loss"][:1], [loss], [lb], "policy")
    gradients(dlp, slack, "policy gradient")
    off = [0, rows // 2, rows]
    got = T.run_preference(zd, t, off, ref, None, 0.1, 0.05, grad)
    loss, lb, margin, mb, dlp, slack = L.preference(want, off, ref, None, 0.1, 0.05)
    T.near(got["margin"][:1], margin, mb, "margin")
    T.near(got["loss"][:1], [loss], [lb], "preference")
    gradients(dlp, slack, "preference gradient")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("size", [2047.0, 2049.0, 1e4, 1e5, 1e6, 1e7, 1e8, 1e9, 1e10, 1e20, 1e30, 1.1e37, 3e38])
@pytest.mark.parametrize("rows,V", [(10, 300), (10, 9001), (130, 9001), (130, 17001), (129, 33000)])
def test_logits_of_any_size(rows, V, size, kind):
    """spans and all but a few columns masked with finite values, rows masked whole, rows far from zero on either side: in one
    piece, in pieces, whole by one workgroup, and where loss and gradient are one workgroup's"""
    g, z, t = T.logits(rows + V, rows, V, kind)
    z = z.double()
    keep = z[:, [V // 5, V // 2, V - 1]]
    for r in range(rows):
        x, sign = z[r], -1.0 if r % 10 < 5 else 1.0
        if r % 5 == 0:
            x[V // 7: V // 3] = sign * size
        elif r % 5 == 1:
            x[:] = sign * size
            x[[V // 5, V // 2, V - 1]] = keep[r]
        elif r % 5 == 2:
            x[:] = sign * size
        elif r % 5 == 3:
            x[::2] = sign * size
        else:
            x += sign * size
    z = z.to(T.KIND[kind])
    for r in range(rows):                                   # a token that the row makes likely
        x = z[r].double().numpy()
        t[r] = g.choice(np.flatnonzero(x >= x.max() - 10))
    old, ref, adv = T.policy_inputs(g, z, t, rows)
    compare(z, t, old, ref, adv, kind)


FAR = [-745.5, -746.0, -800.0, -1e4, -1e9, -1e30, float(torch.finfo(torch.float32).min)]


@pytest.mark.parametrize("rows,V", [(14, 65), (14, 9001), (140, 33000), (602, 65), (602, 9001)])
def test_preference_counts_every_finite_log_probability(rows, V):
    """tokens whose probability is 0 in 64 bits, but not its logarithm, of which the margin is a sum; pairs of up to 256 rows and longer ones"""
    g, z, t = T.logits(rows, rows, V, "f32")
    off, where = ([0, 2, 4, 5, 8, 11, rows - 2] if rows < 150 else [0, rows // 2, rows - 2]), [1, 3, 4, 5, 8, 10, rows - 1]
    for r, far in zip(where, FAR):                          # the last one lies behind the answers
        z[r, t[r]] = far
    inside = np.arange(rows) < off[-1]
    want = L.rows64(z.double().numpy(), t, inside=inside)
    for q in want:
        if q is not None:
            assert q["lp"] > -np.inf
            q["has"] = True
    assert sum(q is not None and q["lp"] < -745 for q in want) >= 6
    lp = T.lp_of(want)
    ref = np.where(lp < -1e6, -3.0, lp + g.randn(rows)).astype(np.float32)
    for beta in (1e-3, 1e-30):
        grad = torch.full((rows, V), 9.0, device="cuda")
        got = T.run_preference(z.cuda(), t, off, ref, None, beta, 0.1, grad)
        loss, lb, margin, mb, dlp, slack = L.preference(want, off, ref, None, beta, 0.1)
        T.near(got["lp"][:rows], lp, T.lp_bound(want), "logprob")
        T.near(got["margin"][:-1], margin, mb, "margin")
        T.near(got["loss"][:1], [loss], [lb], "loss")
        gg = grad.cpu().numpy()
        for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack)):
            T.near(gg[r], x, b, r)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows,V", [(8, 50), (8, 9001), (130, 9001), (130, 17001)])
def test_a_row_that_is_not_a_distribution_hides_behind_no_masked_token(rows, V, bad):
    """row 1: the token's own logit is -inf beside a NaN or +inf, the row's results are NaN; row 2: a token without a column, the row adds nothing, whatever it
    holds; row 4: -inf beside numbers"""
    g, z, t = T.logits(rows, rows, V, "f32")
    z[1, t[1]] = z[4, t[4]] = -np.inf
    z[1, (t[1] + 1) % V] = z[2, 3] = bad
    t[2] = V if rows < 100 else -1
    zd, out = z.cuda(), torch.empty(rows, device="cuda")
    ws, n = T.space(rows, V)
    B.nanospec_token_logprob(B.logit_rows(zd, T.dev(t, torch.int32)), out, ws, n)
    fine = np.ones(rows, bool)
    fine[[1, 2, 4]] = False

    def check(lp):
        assert np.isnan(lp[1]) and np.isneginf(lp[[2, 4]]).all() and np.isfinite(lp[fine]).all()

    check(out.cpu().numpy())
    one, grad = np.ones(rows, np.float32), torch.full((rows, V), 9.0, device="cuda")
    got = T.run_policy(zd, t, -one, -one, one, None, 0.05, grad)
    check(got["lp"][:rows])
    assert np.isnan(got["row"][1]) and (got["row"][[2, 4]] == 0).all() and np.isnan(got["loss"][0])
    assert torch.isnan(grad[1]).any() and (grad[[2, 4]] == 0).all() and torch.isfinite(grad[torch.from_numpy(fine).cuda()]).all()
    got = T.run_preference(zd, t, [0, 1, 2, 4, 7], None, None, 0.1, 0.0, grad)
    check(np.where(np.arange(rows) < 7, got["lp"][:rows], out.cpu().numpy()))
    assert np.isnan(got["margin"][0]) and np.isfinite(got["margin"][1]) and np.isnan(got["loss"][0])
    assert torch.isnan(grad[:2]).any() and torch.isfinite(grad[2:]).all()
    w = one.copy()
    w[1] = 0                                                # and without that row everything is a number
    got = T.run_policy(zd, t, -one, -one, one, w, 0.05, grad)
    assert np.isfinite(got["loss"][0]) and torch.isfinite(grad).all()


@pytest.mark.parametrize("rows,V", [(6, 70), (6, 9001), (600, 70)])
@pytest.mark.parametrize("smoothing,sign", [(0.0, 1), (1.0, -1), (0.0, -1), (1.0, 1), (0.25, 1), (0.25, -1)])
def test_a_margin_without_end(rows, V, smoothing, sign):
    """a reference that gives a token no probability (-inf, as nanospec_token_logprob says it) in one answer of the first pair: the margin is infinite, and the term
    of the loss whose factor is 0 or whose logarithm is that of 1 adds nothing"""
    g, z, t = T.logits(rows, rows, V, "f32")
    off = [0, rows // 2 - 1, rows // 2, rows // 2 + 1, rows]
    ref = np.full(rows, -2.0, np.float32)
    ref[0 if sign > 0 else rows // 2 - 1] = -np.inf
    grad = torch.full((rows, V), 9.0, device="cuda")
    got = T.run_preference(z.cuda(), t, off, ref, None, 0.1, smoothing, grad)
    assert got["margin"][0] == sign * np.inf
    want = L.rows64(z.double().numpy(), t)
    one, ob, margin, mb, dlp, slack = L.preference(want, off, np.where(np.isinf(ref), -2.0, ref), None, 0.1, smoothing)
    T.near(got["margin"][1:2], margin[1:], mb[1:], "margin")
    wrong = smoothing if sign > 0 else 1 - smoothing        # the factor of log sigma(-inf)
    if wrong:
        assert got["loss"][0] == np.inf
    else:                                                   # half of the second pair's loss
        second = ((1 - smoothing) * np.logaddexp(0, -margin[1]) + smoothing * np.logaddexp(0, margin[1])) / 2
        T.near(got["loss"][:1], [second], [ob], "loss")
    half = np.arange(rows) < rows // 2
    slope = smoothing if sign > 0 else smoothing - 1
    dlp[half] = np.where(np.arange(rows) < rows // 2 - 1, 1, -1)[half] * float(np.float32(0.1)) / 2 * slope
    slack[half] = 1e-14
    gg = grad.cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack)):
        T.near(gg[r], x, b, r)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,off", [(2, 7, [0, 1, 2]), (20, 1000, [2, 9, 9, 13, 17]), (40, 9001, [3, 20, 37]), (600, 300, [0, 400, 590]), (150, 17001, [1, 40, 90, 100, 149]),
                                        (130, 33000, [0, 60, 130]), (1300, 33, list(range(0, 1285, 5)))])
def test_preference_without_a_gradient(rows, V, off, kind):
    """the loss, the margins and the log-probabilities alone, as for a validation set; log-probabilities are the same to the last bit as beside a gradient"""
    g, z, t = T.logits(rows + 3 * V, rows, V, kind)
    inside = (np.arange(rows) >= off[0]) & (np.arange(rows) < off[-1])
    zd = z.cuda()
    zd[torch.from_numpy(~inside).cuda()] = float("nan")
    for plain in (True, False):
        w = None if plain else T.weights(g, rows)
        ref = None if plain else (T.lp_of(L.rows64(z.double().numpy(), t)) + g.randn(rows) * 0.4).astype(np.float32)
        want = L.rows64(z.double().numpy(), t, weight=w, inside=inside)
        loss, lb, margin, mb, _, _ = L.preference(want, off, ref, w, 0.2, 0.1)
        got = T.run_preference(zd, t, off, ref, w, 0.2, 0.1, None)
        T.near(got["lp"][:rows], T.lp_of(want), T.lp_bound(want), "logprob")
        T.near(got["margin"][:-1], margin, mb, "margin")
        T.near(got["loss"][:1], [loss], [lb], "loss")
        assert got["loss"][1] == got["margin"][-1] == got["lp"][rows] == 9.0
        beside = T.run_preference(zd, t, off, ref, w, 0.2, 0.1, torch.empty((rows, V), device="cuda"))
        assert np.array_equal(got["lp"], beside["lp"])
        # margins and losses are added by workgroups of another size there
        T.near(beside["margin"][:-1], margin, mb, "margin")
        T.near(beside["loss"][:1], [loss], [lb], "loss")


@pytest.mark.parametrize("rows,V", [(6, 50), (6, 9001), (130, 9001), (300, 50)])
def test_a_ratio_without_end(rows, V):
    """a policy before that gave the token no probability (-inf) or hardly one: with an advantage of 0 the row adds its KL term, with a positive one the clipped term"""
    g, z, t = T.logits(rows, rows, V, "f32")
    old, ref, adv = T.policy_inputs(g, z, t, rows)
    old[:4] = [-np.inf, -900.0, -np.inf, -900.0]
    adv[:4] = [0.0, 0.0, 0.5, 0.5]
    grad = torch.full((rows, V), 9.0, device="cuda")
    got = T.run_policy(z.cuda(), t, old, ref, adv, None, 0.05, grad)
    want = L.rows64(z.double().numpy(), t)
    near_old = old.copy()
    near_old[:4] = np.float32(T.lp_of(want)[:4] - 5)          # a ratio beyond the clip for which the formula needs no limit
    loss, lb, row, rb, dlp, slack = L.policy(want, near_old, ref, adv, None, 0.2, 0.28, 0.05)
    T.near(got["row"][:rows], row, rb, "rows")
    T.near(got["loss"][:1], [loss], [lb], "loss")
    gg = grad.cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack)):
        T.near(gg[r], x, b, r)
    z[1, 0] = np.nan                                        # and a NaN is none of these
    got = T.run_policy(z.cuda(), t, old, ref, adv, None, 0.05, grad)
    assert np.isnan(got["row"][1]) and np.isfinite(np.delete(got["row"][:rows], 1)).all() and np.isnan(got["loss"][0])


def strided(z, kind, lead, wide):
    """z in the columns lead .. of rows of `wide` columns, 7 around it"""
    buf = torch.full((z.shape[0], wide), 7.0, dtype=T.KIND[kind], device="cuda")
    buf[:, lead:lead + z.shape[1]] = z.cuda()
    return buf, buf[:, lead:lead + z.shape[1]]


@pytest.mark.parametrize("kind,grad_kind,inplace", [("f32", "f32", True), ("f32", "bf16", False), ("bf16", "bf16", True), ("bf16", "f32", False)])
@pytest.mark.parametrize("rows,V", [(130, 4099), (128, 17003), (128, 66001), (129, 140003)])
def test_strided_rows_that_one_workgroup_holds(rows, V, kind, grad_kind, inplace):
    """rows that start at odd elements, with columns of others between them: policy loss, preference loss and log-probabilities"""
    g, z, t = T.logits(rows + V, rows, V, kind)
    old, ref, adv = T.policy_inputs(g, z, t, rows)
    w = T.weights(g, rows)
    for loss in ("policy", "preference"):
        buf, view = strided(z, kind, 3, V + 11)
        gbuf, gview = (buf, view) if inplace else strided(torch.zeros_like(z), grad_kind, 5, V + 8)
        if loss == "policy":
            want = L.rows64(z.double().numpy(), t, weight=w)
            got = T.run_policy(view, t, old, ref, adv, w, 0.05, gview)
            total, bound, _, _, dlp, slack = L.policy(want, old, ref, adv, w, 0.2, 0.28, 0.05)
        else:
            off = [2, 50, 60, 61, rows - 3]
            want = L.rows64(z.double().numpy(), t, weight=w, inside=(np.arange(rows) >= 2) & (np.arange(rows) < rows - 3))
            got = T.run_preference(view, t, off, ref, w, 0.2, 0.1, gview)
            total, bound, _, _, dlp, slack = L.preference(want, off, ref, w, 0.2, 0.1)
        T.near(got["lp"][:rows], T.lp_of(want), T.lp_bound(want), "logprob")
        T.near(got["loss"][:1], [total], [bound], "loss")
        gg, lead = gbuf.float().cpu().numpy(), 3 if inplace else 5
        for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 1.0, T.NAME[T.KIND[grad_kind]])):
            T.near(gg[r, lead:lead + V], x, b, r)
        assert (gg[:, :lead] == 7).all() and (gg[:, lead + V:] == 7).all()
        if not inplace:
            assert torch.equal(view, z.cuda()) and (buf[:, :3] == 7).all() and (buf[:, 3 + V:] == 7).all()


@pytest.mark.parametrize("counts,M,off", [([5, 0, 64, 700], 3, [0, 2, 4, 7, 12]), ([2300] * 5, 8, [1, 9, 20, 33, 38]), ([9000, 0, 1, 4100, 8192] * 5, 7, [0, 80, 174]), ([300, 299, 7] * 100, 2, [0, 290, 600]),
                                          ([33000, 20000], 70, [0, 30, 71, 90, 139]), ([1], 1, [0, 1, 1])])
def test_preference_over_active_sets(counts, M, off):
    """pairs of answers on the active sets' logits, with tokens that the sets do not hold; columns behind the live ones are neither read nor written"""
    V, batch = 40009, len(counts)
    g = np.random.RandomState(M + batch)
    cap = (max(counts) + 64) // 64 * 64
    ids = [np.sort(g.permutation(V)[:n]).astype(np.int32) for n in counts]
    lists = np.full((batch, cap), -5, np.int32)
    for b, x in enumerate(ids):
        lists[b, :len(x)] = x
    rows = batch * M
    z = torch.from_numpy((g.randn(rows, cap) * 2).astype(np.float32))
    t = np.array([ids[r // M][g.randint(counts[r // M])] if counts[r // M] and r % 5 != 3 else g.randint(V) for r in range(rows)], np.int32)
    live = [z[r, :counts[r // M]].double().numpy() for r in range(rows)]
    zd = z.cuda()
    for r in range(rows):
        zd[r, counts[r // M]:] = float("nan")
    src = B.logit_rows(zd, T.dev(t, torch.int32), ids=T.dev(lists, torch.int32), n=T.dev(counts, torch.int32), rows_per_list=M)
    inside = (np.arange(rows) >= off[0]) & (np.arange(rows) < off[-1])
    want = L.rows64(live, t, ids=[ids[r // M] for r in range(rows)], inside=inside)
    lp = T.lp_of(want)
    ref = (np.where(np.isfinite(lp), lp, -1.0) + g.randn(rows) * 0.4).astype(np.float32)
    loss, lb, margin, mb, dlp, slack = L.preference(want, off, ref, None, 0.2, 0.1)
    grad = torch.full((rows, cap), 9.0, device="cuda")
    for gr in (grad, None):
        got = T.run_preference(zd, t, off, ref, None, 0.2, 0.1, gr, rows=src)
        T.near(got["lp"][:rows], lp, T.lp_bound(want), "logprob")
        T.near(got["margin"][:-1], margin, mb, "margin")
        T.near(got["loss"][:1], [loss], [lb], "loss")
    gg = grad.cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [len(a) for a in live], dlp, slack)):
        T.near(gg[r, :len(live[r])], x, b, r)
        assert (gg[r, len(live[r]):] == 9.0).all()
    every = L.rows64(live, t, ids=[ids[r // M] for r in range(rows)])
    out = torch.empty(rows, device="cuda")
    ws, n = T.space(rows, cap)
    B.nanospec_token_logprob(src, out, ws, n)
    T.near(out.cpu(), T.lp_of(every), T.lp_bound(every), "logprob of all rows")
