"""Log-probabilities of tokens and the losses on rows of logits, with their gradients, against 64 bits; tolerances are those derived in
losses64.py."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import losses64 as L
from paper_2605_26444_amd import binding as B

pytestmark = pytest.mark.gpu

KIND = {"f32": torch.float32, "bf16": torch.bfloat16}
NAME = {torch.float32: "float32", torch.bfloat16: "bfloat16"}


def space(rows, V):
    n = B.nanospec_loss_workspace(rows, V)
    assert n > 0
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda"), n      # NaN everywhere: nothing may depend on what it held


def dev(x, dtype=torch.float32):
    return torch.as_tensor(np.asarray(x)).to(dtype).cuda()


def logits(seed, rows, V, kind, sigma=2.0):
    g = np.random.RandomState(seed)
    z = torch.from_numpy((g.randn(rows, V) * sigma).astype(np.float32)).to(KIND[kind])
    t = g.randint(0, V, rows).astype(np.int32)
    at = torch.arange(rows), torch.from_numpy(t).long()
    z[at] = (z[at].float() + torch.from_numpy(g.randn(rows).astype(np.float32)) * 3 + 5).to(KIND[kind])
    return g, z, t


def near(got, want, bound, what):
    got, want, bound = np.asarray(got, np.float64), np.asarray(want, np.float64), np.asarray(bound, np.float64)
    special = ~np.isfinite(want)
    assert np.array_equal(got[special], want[special], equal_nan=True), what
    far = np.abs(got[~special] - want[~special]) - np.broadcast_to(bound, want.shape)[~special]
    assert not np.isnan(far).any() and (far.size == 0 or far.max() <= 0), (what, far.max())


def lp_of(rows):
    return np.array([0.0 if q is None else q["lp"] for q in rows])


def lp_bound(rows):
    return np.array([0.0 if q is None or not np.isfinite(q["lp"]) else q["delta"] + L.U * (abs(q["lp"]) + q["delta"]) for q in rows])


SIZES = [(1, 1), (1, 2), (3, 7), (5, 63), (2, 64), (9, 257), (4, 1000), (33, 1023), (2, 4096), (3, 4097), (2, 8191), (7, 32000), (1, 128256), (2500, 33)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", SIZES)
def test_log_probabilities(rows, V, kind):
    g, z, t = logits(rows + V, rows, V, kind)
    out = torch.full((rows + 1,), 9.0, device="cuda")
    ws, n = space(rows, V)
    B.nanospec_token_logprob(B.logit_rows(z.cuda(), dev(t, torch.int32)), out, ws, n)
    want = L.rows64(z.double().numpy(), t)
    near(out[:rows].cpu(), lp_of(want), lp_bound(want), "logprob")
    assert out[rows] == 9.0


def weights(g, rows):
    w = g.rand(rows).astype(np.float32) + 0.1
    w[g.rand(rows) < 0.25] = 0
    if rows > 2:
        w[1] = 0
        w[2] = -0.5
    return w


def policy_inputs(g, z, t, rows):
    lp = lp_of(L.rows64(z.double().numpy(), t))
    old, ref, adv = lp + g.randn(rows) * 0.25, lp + g.randn(rows) * 0.5, g.randn(rows)
    return [x.astype(np.float32) for x in (old, ref, adv)]


def run_policy(z, t, old, ref, adv, w, beta, grad, scale=1.0, rows=None, lo=0.2, hi=0.28):
    R, V = z.shape
    out = {k: torch.full((n,), 9.0, device="cuda") for k, n in (("loss", 2), ("row", R + 1), ("lp", R + 1))}
    ws, n = space(R, V)
    B.nanospec_policy_loss(rows or B.logit_rows(z, dev(t, torch.int32)), dev(old), None if ref is None else dev(ref), dev(adv), None if w is None else dev(w), lo, hi, beta,
                           out["loss"], out["row"], out["lp"], grad, ws, n, grad_scale=scale)
    return {k: v.cpu().numpy() for k, v in out.items()}


@pytest.mark.parametrize("grad_kind", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", SIZES)
def test_policy(rows, V, kind, grad_kind):
    g, z, t = logits(3 * rows + V, rows, V, kind)
    old, ref, adv = policy_inputs(g, z, t, rows)
    w = weights(g, rows)
    zd = z.cuda()
    if rows > 2:
        zd[1] = float("nan")                                              # rows that do not count may hold anything
        old[1] = np.nan
    grad = torch.full((rows + 1, V), 9.0, dtype=KIND[grad_kind], device="cuda")
    got = run_policy(zd, t, old, ref, adv, w, 0.05, grad, scale=3.0)
    want = L.rows64(z.double().numpy(), t, weight=w)
    loss, lb, row, rb, dlp, slack = L.policy(want, old, ref, adv, w, 0.2, 0.28, 0.05)
    near(got["lp"][:rows], lp_of(want), lp_bound(want), "logprob")
    near(got["row"][:rows], row, rb, "rows")
    near(got["loss"][:1], [loss], [lb], "loss")
    assert got["loss"][1] == got["row"][rows] == got["lp"][rows] == 9.0
    gg = grad.float().cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 3.0, NAME[KIND[grad_kind]])):
        near(gg[r], x, b, r)
    assert (gg[rows] == 9.0).all()


MANY = [(128, 4096), (129, 4097), (131, 4103), (128, 9001), (150, 17001), (130, 33000), (128, 66003), (129, 131072), (128, 140001), (300, 5000)]


@pytest.mark.parametrize("kind,grad_kind,inplace", [("f32", "f32", False), ("f32", "f32", True), ("f32", "bf16", False), ("bf16", "bf16", False), ("bf16", "bf16", True), ("bf16", "f32", False)])
@pytest.mark.parametrize("rows,V", MANY)
def test_policy_on_many_long_rows(rows, V, kind, grad_kind, inplace):
    """rows that one workgroup holds: its registers, its LDS, what it streams, and every kind of end"""
    g, z, t = logits(rows + V, rows, V, kind)
    t[3], t[4], t[5], t[6] = 0, V - 1, -1, V // 2
    z[7, t[7]] = -np.inf
    z[8] = -np.inf
    z[9, V // 3:] = float(torch.finfo(KIND[kind]).min)
    z[10, ::2] = -np.inf
    t[10] = 1
    lp = lp_of(L.rows64(z.double().numpy(), t))
    lp = np.where(np.isfinite(lp) & (lp > -700), lp, -2.0)
    old, ref, adv = [(lp + g.randn(rows) * s).astype(np.float32) for s in (0.25, 0.5)] + [g.randn(rows).astype(np.float32)]
    w = weights(g, rows)
    w[3:11] = 0.5
    zd = z.cuda()
    zd[1], old[1] = float("nan"), np.nan
    want = L.rows64(z.double().numpy(), t, weight=w)
    loss, lb, row, rb, dlp, slack = L.policy(want, old, ref, adv, w, 0.2, 0.28, 0.05)
    grad = zd if inplace else torch.full((rows + 1, V), 9.0, dtype=KIND[grad_kind], device="cuda")
    got = run_policy(zd, t, old, ref, adv, w, 0.05, grad, scale=2.0)
    near(got["lp"][:rows], lp_of(want), lp_bound(want), "logprob")
    near(got["row"][:rows], row, rb, "rows")
    near(got["loss"][:1], [loss], [lb], "loss")
    gg = grad.float().cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 2.0, NAME[KIND[grad_kind]])):
        near(gg[r], x, b, r)
    assert inplace or (gg[rows] == 9.0).all()
    out = torch.empty(rows, device="cuda")
    ws, n = space(rows, V)
    zd = z.cuda()
    B.nanospec_token_logprob(B.logit_rows(zd, dev(t, torch.int32)), out, ws, n)
    everything = L.rows64(z.double().numpy(), t)
    near(out.cpu(), lp_of(everything), lp_bound(everything), "logprob")


@pytest.mark.parametrize("rows,V,off", [(150, 17001, [1, 40, 90, 100, 149]), (260, 40000, [0, 100, 255]), (129, 5000, [0, 1, 2, 3, 129]), (128, 70001, [5, 60, 128])])
@pytest.mark.parametrize("kind,grad_kind", [("f32", "f32"), ("bf16", "bf16")])
def test_preference_on_many_long_rows(rows, V, off, kind, grad_kind):
    test_preference(rows, V, off, kind, grad_kind, False)


@pytest.mark.parametrize("V", [63, 1000, 32001])
def test_policy_without_weights_reference_and_gradient(V):
    rows = 6
    g, z, t = logits(V, rows, V, "f32")
    old, ref, adv = policy_inputs(g, z, t, rows)
    got = run_policy(z.cuda(), t, old, None, adv, None, 0.0, None)
    want = L.rows64(z.double().numpy(), t)
    loss, lb, row, rb, _, _ = L.policy(want, old, None, adv, None, 0.2, 0.28, 0.0)
    near(got["row"][:rows], row, rb, "rows")
    near(got["loss"][:1], [loss], [lb], "loss")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_policy_on_strided_rows_and_in_place(kind):
    rows, V, wide = 9, 1001, 1205
    g, z, t = logits(5, rows, V, kind)
    old, ref, adv = policy_inputs(g, z, t, rows)
    want = L.rows64(z.double().numpy(), t)
    _, _, _, _, dlp, slack = L.policy(want, old, ref, adv, None, 0.2, 0.28, 0.1)
    buf = torch.full((rows, wide), 7.0, dtype=KIND[kind], device="cuda")
    buf[:, 3:3 + V] = z.cuda()
    view = buf[:, 3:3 + V]
    run_policy(view, t, old, ref, adv, None, 0.1, view)
    gg = buf.float().cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 1.0, NAME[KIND[kind]])):
        near(gg[r, 3:3 + V], x, b, r)
    assert (gg[:, :3] == 7).all() and (gg[:, 3 + V:] == 7).all()


@pytest.mark.parametrize("V", [40, 5000])
def test_masks_infinities_and_tokens_without_a_probability(V):
    rows = 12
    low = float(torch.finfo(torch.float32).min)
    g, z, t = logits(11, rows, V, "f32")
    z[0] = -np.inf                                                         # a row without any probability
    z[1, : V // 2] = -np.inf
    t[1] = V - 1
    z[2] = low                                                             # masked to the lowest value everywhere: all the same
    z[3, V // 2:] = low
    t[3] = V - 2                                                           # a masked token
    t[4], t[5], t[6] = -1, V, 2 ** 31 - 1                                  # padding and ids outside
    z[7, t[7]] = -np.inf
    z[8, :] = -np.inf
    z[8, t[8]] = 3.0                                                       # the only one left: probability one
    z[9, 0], z[10, 1] = np.nan, np.inf
    z[11] *= 40                                                            # a sharp row
    lp = lp_of(L.rows64(z.double().numpy(), t))
    safe = np.where(np.isfinite(lp) & (lp > -700), lp, -3.0)
    old, ref, adv = [(safe + d).astype(np.float32) for d in (0.1, -0.2)] + [np.linspace(-1, 1, rows).astype(np.float32)]
    out = torch.empty(rows, device="cuda")
    ws, n = space(rows, V)
    B.nanospec_token_logprob(B.logit_rows(z.cuda(), dev(t, torch.int32)), out, ws, n)
    want = L.rows64(z.double().numpy(), t)
    near(out.cpu(), lp_of(want), lp_bound(want), "logprob")
    assert np.isneginf(out.cpu().numpy()[[0, 4, 5, 6, 7]]).all() and np.isnan(out.cpu().numpy()[[9, 10]]).all()
    for keep_nan in (False, True):
        w = np.ones(rows, np.float32)
        if not keep_nan:
            w[9:11] = 0
        grad = torch.full((rows, V), 9.0, device="cuda")
        got = run_policy(z.cuda(), t, old, ref, adv, w, 0.05, grad)
        want = L.rows64(z.double().numpy(), t, weight=w)
        loss, lb, row, rb, dlp, slack = L.policy(want, old, ref, adv, w, 0.2, 0.28, 0.05)
        gg = grad.cpu().numpy()
        for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack)):
            if keep_nan and r in (9, 10):
                assert np.isnan(gg[r]).any() and np.isnan(got["row"][r])
            else:
                near(gg[r], x, b, r)
                near(got["row"][r], row[r], rb[r], r)
        if keep_nan:
            assert np.isnan(got["loss"][0])
        else:
            near(got["loss"][:1], [loss], [lb], "loss")


def run_preference(z, t, off, ref, w, beta, smoothing, grad, scale=1.0, rows=None):
    R, V = z.shape
    out = {k: torch.full((n,), 9.0, device="cuda") for k, n in (("loss", 2), ("margin", len(off) // 2 + 1), ("lp", R + 1))}
    ws, n = space(R, V)
    B.nanospec_preference_loss(rows or B.logit_rows(z, dev(t, torch.int32)), off, None if ref is None else dev(ref), None if w is None else dev(w), beta, smoothing, out["loss"],
                               out["margin"], out["lp"], grad, ws, n, grad_scale=scale)
    return {k: v.cpu().numpy() for k, v in out.items()}


OFFSETS = [(2, 7, [0, 1, 2]), (20, 63, [0, 11, 20]), (20, 1000, [2, 9, 9, 13, 17]), (30, 4097, [0, 5, 10, 11, 20, 20, 30]), (9, 32000, [1, 4, 8]), (4, 16, [2, 2, 2]),
           (1300, 33, list(range(0, 1285, 5))), (40, 9000, [3, 20, 37])]


@pytest.mark.parametrize("kind,grad_kind", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,V,off", OFFSETS)
@pytest.mark.parametrize("plain", [False, True])
def test_preference(rows, V, off, kind, grad_kind, plain):
    g, z, t = logits(rows + 7 * V, rows, V, kind)
    inside = (np.arange(rows) >= off[0]) & (np.arange(rows) < off[-1])
    w = None if plain else weights(g, rows)
    ref = None if plain else (lp_of(L.rows64(z.double().numpy(), t)) + g.randn(rows) * 0.4).astype(np.float32)
    zd = z.cuda()
    zd[torch.from_numpy(~inside).cuda()] = float("nan")
    grad = torch.full((rows + 1, V), 9.0, dtype=KIND[grad_kind], device="cuda")
    got = run_preference(zd, t, off, ref, w, 0.2, 0.1, grad, scale=0.5)
    want = L.rows64(z.double().numpy(), t, weight=w, inside=inside)
    loss, lb, margin, mb, dlp, slack = L.preference(want, off, ref, w, 0.2, 0.1)
    near(got["lp"][:rows], lp_of(want), lp_bound(want), "logprob")
    near(got["margin"][:-1], margin, mb, "margin")
    near(got["loss"][:1], [loss], [lb], "loss")
    assert got["loss"][1] == got["margin"][-1] == got["lp"][rows] == 9.0
    gg = grad.float().cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 0.5, NAME[KIND[grad_kind]])):
        near(gg[r], x, b, r)
    assert (gg[rows] == 9.0).all()


@pytest.mark.parametrize("rows,V,off", [(600, 9000, [0, 400, 590]), (300, 100, [0, 270, 300]), (258, 20000, [0, 257, 258]), (40, 5001, [1, 15, 33])])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_preference_on_long_answers_and_in_place(rows, V, off, kind):
    g, z, t = logits(rows + V, rows, V, kind)
    inside = (np.arange(rows) >= off[0]) & (np.arange(rows) < off[-1])
    w = weights(g, rows)
    ref = (lp_of(L.rows64(z.double().numpy(), t)) + g.randn(rows) * 0.4).astype(np.float32)
    zd = z.cuda()
    got = run_preference(zd, t, off, ref, w, 0.02, 0.1, zd)
    want = L.rows64(z.double().numpy(), t, weight=w, inside=inside)
    loss, lb, margin, mb, dlp, slack = L.preference(want, off, ref, w, 0.02, 0.1)
    near(got["margin"][:-1], margin, mb, "margin")
    near(got["loss"][:1], [loss], [lb], "loss")
    gg = zd.float().cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [V] * rows, dlp, slack, 1.0, NAME[KIND[kind]])):
        near(gg[r], x, b, r)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_more_logits_than_32_bits_count(kind):
    rows, V = 17000, 128256
    z = torch.zeros((rows, V), dtype=KIND[kind], device="cuda")
    some = [0, 1, 8371, 8372, 16743, 16744, 16745, rows - 1]                # around 2^30 and 2^31 elements
    g, zs, ts = logits(3, len(some), V, kind)
    z[torch.tensor(some).cuda()] = zs.cuda()
    t = np.full(rows, 7, np.int32)
    t[some] = ts
    lp = lp_of(L.rows64(zs.double().numpy(), ts))
    old, ref, adv = (np.full(rows, -np.log(V), np.float32) for _ in range(3))
    old[some], ref[some], adv[some] = lp + 0.1, lp - 0.2, g.randn(len(some))
    got = run_policy(z, t, old, ref, adv, None, 0.05, z)
    want = L.rows64(zs.double().numpy(), ts)
    _, _, row, rb, dlp, slack = L.policy(want, old[some], ref[some], adv[some], None, 0.2, 0.28, 0.05)
    near(got["lp"][some], lp_of(want), lp_bound(want), "logprob")
    near(got["row"][some], row, rb, "rows")
    for r, (x, b) in zip(some, L.gradient(want, [V] * len(some), dlp, slack, 1.0, NAME[KIND[kind]])):
        near(z[r].float().cpu(), x, b, r)
    flat = np.delete(got["lp"][:rows], some)
    assert np.abs(flat + np.log(V)).max() < 1e-5


def test_on_a_stream_of_the_callers():
    rows, V = 60, 3001
    g, z, t = logits(4, rows, V, "f32")
    zd, td, fresh = torch.zeros((rows, V), device="cuda"), dev(t, torch.int32), z.cuda()
    out = torch.zeros(rows, device="cuda")
    ws, n = space(rows, V)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy = torch.zeros(1 << 28, device="cuda").add_(1).add_(1)
        zd.copy_(fresh)
    B.nanospec_token_logprob(B.logit_rows(zd, td), out, ws, n, stream=side)
    with torch.cuda.stream(side):
        copy = out.clone()
    side.synchronize()
    want = L.rows64(z.double().numpy(), t)
    near(copy.cpu(), lp_of(want), lp_bound(want), "logprob")
    assert busy[0] == 2


def test_a_far_margin_neither_overflows_nor_loses_the_gradient():
    z = torch.tensor([[0.0, 300.0], [0.0, 0.0], [0.0, 0.0], [0.0, 300.0]])
    t = np.zeros(4, np.int32)
    grad = torch.empty((4, 2), device="cuda")
    got = run_preference(z.cuda(), t, [0, 1, 2, 3, 4], None, None, 10.0, 0.0, grad)
    want = L.rows64(z.double().numpy(), t)
    loss, lb, margin, mb, dlp, slack = L.preference(want, [0, 1, 2, 3, 4], None, None, 10.0, 0.0)
    near(got["margin"][:2], margin, mb, "margin")
    near(got["loss"][:1], [loss], [lb], "loss")
    for r, (x, b) in enumerate(L.gradient(want, [2] * 4, dlp, slack)):
        near(grad[r].cpu(), x, b, r)


@pytest.mark.parametrize("counts,M", [([5, 0, 64, 700], 3), ([1], 4), ([2300] * 5, 8), ([9000, 4096], 2), ([9000, 0, 1, 4100, 8192] * 5, 7)])
def test_on_the_active_sets_of_a_state(counts, M):
    V, batch = 20011, len(counts)
    g = np.random.RandomState(M)
    st = B.State(V, 16, batch, 1, max(counts), M, 1)
    ids = [np.sort(g.permutation(V)[:n]).astype(np.int32) for n in counts]
    off = np.zeros(batch + 1, np.int32)
    off[1:] = np.cumsum(counts)
    B.nanospec_vocab_init(st.h, None, np.zeros(batch + 1, np.int32), dev(np.concatenate(ids), torch.int32), off)
    cap, rows = st.capacity, batch * M
    z = torch.from_numpy((g.randn(rows, cap) * 2).astype(np.float32))
    t = np.array([ids[r // M][g.randint(counts[r // M])] if counts[r // M] and r % 5 != 3 else g.randint(V) for r in range(rows)], np.int32)
    live = [z[r, :counts[r // M]].double().numpy() for r in range(rows)]
    zd = z.cuda()
    for r in range(rows):
        zd[r, counts[r // M]:] = float("nan")                              # behind the live columns: neither read nor written
    lists = [ids[r // M] for r in range(rows)]
    src = B.logit_rows(zd, dev(t, torch.int32), V=cap, ids=st.ids_ptr, n=st.n_ptr, rows_per_list=M)
    out = torch.empty(rows, device="cuda")
    ws, n = space(rows, cap)
    B.nanospec_token_logprob(src, out, ws, n)
    want = L.rows64(live, t, ids=lists)
    near(out.cpu(), lp_of(want), lp_bound(want), "logprob")
    lp = np.where(np.isfinite(lp_of(want)), lp_of(want), -1.0)
    old, ref, adv = [(lp + g.randn(rows) * s).astype(np.float32) for s in (0.2, 0.4)] + [g.randn(rows).astype(np.float32)]
    grad = torch.full((rows, cap), 9.0, device="cuda")
    got = run_policy(zd, t, old, ref, adv, None, 0.05, grad, rows=src)
    loss, lb, row, rb, dlp, slack = L.policy(want, old, ref, adv, None, 0.2, 0.28, 0.05)
    near(got["row"][:rows], row, rb, "rows")
    near(got["loss"][:1], [loss], [lb], "loss")
    gg = grad.cpu().numpy()
    for r, (x, b) in enumerate(L.gradient(want, [len(a) for a in live], dlp, slack)):
        near(gg[r, :len(live[r])], x, b, r)
        assert (gg[r, len(live[r]):] == 9.0).all()
    st.close()


@pytest.mark.parametrize("rows", [40, 200, 700])
def test_captured_and_replayed(rows):
    """a training step's three calls in a graph, replayed against new inputs with eager work between"""
    V = 9001
    g, z, t = logits(21, rows, V, "f32")
    old, ref, adv = policy_inputs(g, z, t, rows)
    w = weights(g, rows)
    zd, td, args = z.cuda(), dev(t, torch.int32), [dev(x) for x in (old, ref, adv, w)]
    outs = [{"loss": torch.zeros(1, device="cuda"), "grad": torch.zeros((rows, V), device="cuda"), "lp": torch.zeros(rows, device="cuda")} for _ in range(2)]
    spaces = [space(rows, V) for _ in range(2)]
    off = [0, 9, 19, 28, rows]

    def both(o, s):
        src = B.logit_rows(zd, td)
        B.nanospec_policy_loss(src, *args, 0.2, 0.28, 0.05, o["loss"], None, o["lp"], o["grad"], *s)
        B.nanospec_preference_loss(src, off, args[1], args[3], 0.1, 0.05, o["loss"], None, None, o["grad"], *s)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    both(outs[0], spaces[0])
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        both(outs[0], spaces[0])
    for turn in range(3):
        zd.copy_(logits(30 + turn, rows, V, "f32")[1])
        both(outs[1], spaces[1])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in outs[0]:
            assert torch.equal(outs[0][k], outs[1][k]), (turn, k)


def test_results_do_not_change_from_run_to_run():
    rows, V = 300, 50001
    g, z, t = logits(31, rows, V, "bf16")
    old, ref, adv = policy_inputs(g, z, t, rows)
    zd = z.cuda()
    first = None
    for _ in range(4):
        grad = torch.empty((rows, V), dtype=torch.bfloat16, device="cuda")
        got = run_policy(zd, t, old, ref, adv, None, 0.05, grad)
        now = [grad.view(torch.int16).cpu().numpy()] + list(got.values())
        assert first is None or all(np.array_equal(a, b) for a, b in zip(first, now))
        first = now


def test_refusals():
    rows, V = 4, 32
    lib = B.lib()
    z, t = torch.zeros((rows, V), device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    f, grad = torch.zeros(16, device="cuda"), torch.full((rows, 2 * V), 9.0, device="cuda")
    ws, n = space(rows, V)
    p = lambda x, o=0: C.c_void_p(x.data_ptr() + o)
    src = lambda **k: (lambda r: [setattr(r, a, b) for a, b in k.items()] and r or r)(B.logit_rows(z, t))

    def policy(rows_=None, **k):
        a = dict(old=p(f), ref=p(f), adv=p(f), w=None, lo=0.2, hi=0.2, kl=0.1, loss=p(f), grad=None, kind=B.F32, ld=V, scale=1.0, ws=p(ws), n=n)
        a.update(k)
        return lib.nanospec_policy_loss(rows_ if rows_ is not None else src(), a["old"], a["ref"], a["adv"], a["w"], a["lo"], a["hi"], a["kl"], a["loss"], None, None, a["grad"],
                                        a["kind"], a["ld"], a["scale"], a["ws"], a["n"], None)

    def pair(off, rows_=None, pairs=None, **k):
        a = dict(ref=None, w=None, beta=0.1, e=0.0, loss=p(f), grad=None, kind=B.F32, ld=V, scale=1.0, ws=p(ws), n=n)
        a.update(k)
        o = None if off is None else np.asarray(off, np.int32)
        return lib.nanospec_preference_loss(rows_ if rows_ is not None else src(), None if o is None else o.ctypes.data, len(o) // 2 if pairs is None else pairs, a["ref"], a["w"],
                                            a["beta"], a["e"], a["loss"], None, None, a["grad"], a["kind"], a["ld"], a["scale"], a["ws"], a["n"], None)

    assert policy() == B.OK and pair([0, 2, 4]) == B.OK
    nan = float("nan")
    bad_rows = [dict(d_logits=None), dict(d_tokens=None), dict(rows=0), dict(rows=-1), dict(V=0), dict(V=2 ** 30 + 1), dict(ld=V - 1), dict(ld=2 ** 60), dict(type=2), dict(type=-1),
                dict(d_ids=t.data_ptr()), dict(d_n=t.data_ptr()), dict(d_ids=t.data_ptr(), d_n=t.data_ptr(), rows_per_list=0)]
    for k in bad_rows:
        assert policy(src(**k)) == B.EINVAL, k
        assert pair([0, 2, 4], src(**k)) == B.EINVAL, k
        assert lib.nanospec_token_logprob(src(**k), p(f), p(ws), n, None) == B.EINVAL, k
    assert lib.nanospec_token_logprob(None, p(f), p(ws), n, None) == B.EINVAL and lib.nanospec_token_logprob(src(), None, p(ws), n, None) == B.EINVAL
    assert lib.nanospec_token_logprob(src(), p(f), None, n, None) == B.EINVAL and lib.nanospec_token_logprob(src(), p(f), p(ws), n - 1, None) == B.ECAPACITY
    for k in (dict(old=None), dict(adv=None), dict(loss=None), dict(ref=None), dict(lo=-0.1), dict(hi=-1.0), dict(lo=nan), dict(hi=nan), dict(kl=nan), dict(scale=nan), dict(ws=None),
              dict(ws=p(ws, 8)), dict(grad=p(grad), kind=7), dict(grad=p(grad), ld=V - 1), dict(grad=p(z), kind=B.BF16), dict(grad=p(z), ld=V + 1), dict(grad=p(z, 4)),
              dict(grad=p(z, 4 * V))):
        assert policy(**k) == B.EINVAL, k
    assert policy(n=n - 1) == B.ECAPACITY and policy(grad=p(z)) == B.OK and policy(ref=None, kl=0.0) == B.OK
    for off in ([0, 3, 2], [-1, 2, 4], [0, 2, 5]):
        assert pair(off) == B.EINVAL, off
    assert pair(None, pairs=1) == B.EINVAL and pair([0, 2, 4], pairs=0) == B.EINVAL
    assert pair([0] * 259) == B.ECAPACITY and pair([0] * 257) == B.OK
    for k in (dict(beta=nan), dict(e=-0.1), dict(e=1.1), dict(e=nan), dict(loss=None), dict(ws=None), dict(grad=p(z), ld=V + 1), dict(scale=nan)):
        assert pair([0, 2, 4], **k) == B.EINVAL, k
    assert pair([0, 2, 4], n=n - 1) == B.ECAPACITY
    assert B.nanospec_loss_workspace(0, 5) == -1 and B.nanospec_loss_workspace(5, 0) == -1
    torch.cuda.synchronize()
    assert (grad == 9.0).all()
    for bad in (torch.zeros((4, 4), dtype=torch.float16, device="cuda"), torch.zeros((4, 8), device="cuda")[:, ::2], torch.zeros(8, device="cuda")):
        with pytest.raises(ValueError):
            B.logit_rows(bad, t)
    with pytest.raises(ValueError):
        B.logit_rows(z, t.long())


def test_a_training_step_against_a_reference_head_in_8_bits():
    """the operators as they are used together: the frozen head in 8 bits gives the reference's log-probabilities, the trained head's
    logits the old ones and, after a step along the gradient, the loss that fell as far as the gradient says"""
    V, d, M = 1501, 256, 24
    g = np.random.RandomState(5)
    W = torch.from_numpy((g.randn(V, d) * 0.08).astype(np.float32)).bfloat16().cuda()
    H = torch.from_numpy(g.randn(M, d).astype(np.float32)).bfloat16().cuda()
    t = dev(g.randint(0, V, M), torch.int32)
    q, s = torch.empty((V, d), dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    B.nanospec_quantize_rows(W, V, d, q, s)
    hw = torch.empty(B.nanospec_head_i8_workspace(M, d), dtype=torch.uint8, device="cuda")
    zr, z = torch.empty((M, V), device="cuda"), torch.empty((M, V), device="cuda")
    B.nanospec_dense_head_i8(q, s, H, V, d, M, zr, hw, hw.numel())
    B.nanospec_dense_head(W, H, V, d, M, z)
    ws, n = space(M, V)
    ref, old, lp = (torch.empty(M, device="cuda") for _ in range(3))
    B.nanospec_token_logprob(B.logit_rows(zr, t), ref, ws, n)
    B.nanospec_token_logprob(B.logit_rows(z, t), old, ws, n)
    # both heads' logits are off by their quantization only: a step of 1 / 254 of a row's largest element on either side, d products
    hf, wf = H.float().abs().amax(1), W.float().abs().amax(1)
    far = (hf[:, None] * W.float().abs().sum(1) + wf * H.float().abs().sum(1)[:, None] + d * hf[:, None] * wf / 254) / 254
    assert ((zr - z).abs() <= far * 1.01 + 1e-5).all()
    assert ((ref - old).abs() <= 2 * far.amax(1) * 1.01 + 1e-4).all()
    adv = dev(g.randn(M))
    loss, grad = torch.empty(1, device="cuda"), torch.empty((M, V), device="cuda")
    call = lambda zz, gr: (B.nanospec_policy_loss(B.logit_rows(zz, t), old, ref, adv, None, 0.2, 0.28, 0.05, loss, None, lp, gr, ws, n), float(loss))[1]
    before = call(z, grad)
    assert torch.equal(lp, old)
    h = 2.0 ** -6
    slope = (call(z + h * grad, None) - call(z - h * grad, None)) / (2 * h)
    want = float((grad.double() ** 2).sum())
    # the losses are off by 24 rows of 2^-21 each, over 2 h; the third derivative along the gradient is within 8 |grad|^3
    assert abs(slope - want) <= 24 * 2.0 ** -21 / h + 8 * want ** 1.5 * h * h, (slope, want)
    assert before == call(z, None)
