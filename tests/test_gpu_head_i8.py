"""Rows in 8 bits and the heads on them against the definition: q is what exact arithmetic gives, the sums are integers, so the
logits are known to the last bit -- float32(sum) * (scale_w * scale_h), three roundings in this order."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2605_26444_amd import binding as B
from paper_2605_26444_amd import synth

pytestmark = pytest.mark.gpu


def rows_bf16(seed, rows, d, sigma=1.0):
    return torch.from_numpy(synth.normal_bf16(seed, 0, (rows, d), sigma, threads=1).view(np.int16)).view(torch.bfloat16)


def quantized(x):
    """(q int8, scale float32) of bf16 rows in exact arithmetic: 127 x has 15 bits, its quotient in float64 rounds as the real one"""
    x = x.double().numpy()
    top = np.abs(x).max(axis=1)
    fine = np.isfinite(top)
    with np.errstate(all="ignore"):
        q = np.where((fine & (top > 0))[:, None], np.rint(127.0 * x / top[:, None]), 0.0)
        scale = np.where(fine, top, np.nan).astype(np.float32) / np.float32(127)
    return q.astype(np.int8), scale


def expected(qw, sw, qh, sh):
    """logits [M][V] of quantized rows"""
    total = (torch.from_numpy(qh).cuda().double() @ torch.from_numpy(qw).cuda().double().t()).cpu().numpy()
    assert np.abs(total).max(initial=0) < 2 ** 31
    with np.errstate(all="ignore"):
        return total.astype(np.float32) * (sw[None, :] * sh[:, None])


def workspace(rows, d):
    n = B.nanospec_head_i8_workspace(rows, d)
    assert n > 0
    return torch.empty(n, dtype=torch.uint8, device="cuda"), n


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def special_rows(d):
    big = torch.finfo(torch.bfloat16).max
    out = []
    for f in (lambda i: i * 0.0, lambda i: (i == d - 1) * -2.0, lambda i: i * 0 + 127.0, lambda i: (i % 255 - 127) * 0.5, lambda i: (i % 127 + 0.5) * 2.0 ** 100,
              lambda i: (i % 3 - 1.0) * big, lambda i: (i % 5 - 2) * 2.0 ** -133, lambda i: (i % 5 - 2) * 2.0 ** -126, lambda i: (i == 0) * big + (i == 1) * 2.0 ** -130,
              lambda i: torch.where(i == 3, float("inf"), 1.0), lambda i: torch.where(i == d - 1, float("nan"), 0.5),
              lambda i: torch.where(i == 0, float("-inf"), 0.0)):
        out.append(f(torch.arange(d).double()).to(torch.bfloat16))
    return torch.stack(out)


@pytest.mark.parametrize("rows,d", [(1, 16), (3, 48), (1000, 512), (7, 4112), (65, 1040), (2, 133136)])
def test_rows_are_rounded_as_exact_arithmetic_rounds_them(rows, d):
    x = torch.cat([rows_bf16(rows + d, rows, d, 0.02), special_rows(d)])
    n = len(x)
    q = torch.full((n + 1, d), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((n + 1,), -7.0, device="cuda")
    B.nanospec_quantize_rows(x.cuda(), n, d, q, scale)
    eq, es = quantized(x)
    assert np.array_equal(q.cpu().numpy()[:n], eq)
    assert same(scale.cpu().numpy()[:n], es)
    assert (q[n] == 99).all() and scale[n] == -7.0


@pytest.mark.parametrize("exponent", [0, -133 + 11, 120, -70, -63, -64])
def test_every_quotient_of_two_numbers(exponent):
    """for every mantissa of the largest magnitude a row with every mantissa at every exponent that does not round to 0, and both signs"""
    x = (np.arange(128, 256)[None, :] * 2.0 ** -np.arange(0, 10)[:, None]).ravel()
    x = np.concatenate([x, -x])
    rows = np.stack([np.concatenate([np.where(np.abs(x) <= a, x, 0.0), [a] * 16]) for a in range(128, 256)]) * 2.0 ** exponent
    t = torch.from_numpy(rows).to(torch.bfloat16)
    n, d = t.shape
    q, scale = torch.empty((n, d), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    B.nanospec_quantize_rows(t.cuda(), n, d, q, scale)
    eq, es = quantized(t)
    assert np.array_equal(q.cpu().numpy(), eq) and same(scale.cpu().numpy(), es)
    # and as hidden rows, by the kernels that round them themselves: an identity matrix gives q back
    eye = torch.eye(d, dtype=torch.int8, device="cuda")
    for M in (1, 3, 8, 16):
        out = torch.empty((M, d), device="cuda")
        ws, k = workspace(M, d)
        B.nanospec_dense_head_i8(eye, torch.ones(d, device="cuda"), t[:M].cuda(), d, d, M, out, ws, k)
        assert same(out.cpu().numpy(), eq[:M].astype(np.float32) * es[:M, None])


@pytest.mark.parametrize("V,d", [(1, 16), (17, 48), (100, 256), (1000, 512), (513, 1040), (300, 4096), (5003, 128), (260, 8192)])
@pytest.mark.parametrize("M", [1, 3, 8, 9, 16, 17, 33, 64, 65, 130, 300])
def test_dense_logits_to_the_last_bit(V, d, M):
    w, h = rows_bf16(1, V, d, 0.02), rows_bf16(2, M, d)
    if M > 3:
        h[1] = 0
        h[M - 1, d - 1] = float("nan")
    (qw, sw), (qh, sh) = quantized(w), quantized(h)
    out = torch.full((M + 1, V), 5.0, device="cuda")
    ws, n = workspace(M, d)
    B.nanospec_dense_head_i8(torch.from_numpy(qw).cuda(), torch.from_numpy(sw).cuda(), h.cuda(), V, d, M, out, ws, n)
    got = out.cpu().numpy()
    assert same(got[:M], expected(qw, sw, qh, sh))
    assert (got[M] == 5.0).all()


@pytest.mark.parametrize("V,d,M", [(260, 16384, 1), (260, 16384, 8), (260, 16384, 9), (99, 12304, 5), (99, 8208, 16), (5000, 2064, 12), (40000, 2048, 8), (20011, 4096, 16), (20011, 4080, 3),
                                   (100, 16400, 4), (3001, 4224, 140), (9000, 4112, 700), (2500, 640, 1024)])
def test_dense_logits_of_other_shapes_to_the_last_bit(V, d, M):
    test_dense_logits_to_the_last_bit(V, d, M)


@pytest.mark.parametrize("M", [2, 20, 200])
def test_rows_beyond_the_second_gigabyte(M):
    """V d just below 2^32 bytes: rows at both ends and around 2^31"""
    V, d = 1048575, 4096
    w = torch.zeros((V, d), dtype=torch.int8, device="cuda")
    where = torch.tensor([0, 1, 2 ** 19 - 1, 2 ** 19, 2 ** 19 + 1, V - 300, V - 2, V - 1])
    some = torch.from_numpy(synth.rand_int(9, 0, 0, len(where) * d, -127, 127).reshape(-1, d).astype(np.int8))
    w[where.cuda()] = some.cuda()
    scale = torch.ones(V, device="cuda")
    h = rows_bf16(10, M, d)
    out = torch.full((M, V), 5.0, device="cuda")
    ws, n = workspace(M, d)
    B.nanospec_dense_head_i8(w, scale, h.cuda(), V, d, M, out, ws, n)
    qh, sh = quantized(h)
    assert same(out[:, where.cuda()].cpu().numpy(), expected(some.numpy(), np.ones(len(where), np.float32), qh, sh))
    out[:, where.cuda()] = 0
    assert not out.any()


def test_as_many_sequences_as_a_state_holds():
    test_active_rows_to_the_last_bit([(7 * b) % 40 for b in range(256)], None, 2, 64)


@pytest.mark.parametrize("M", [3, 40])
def test_on_a_stream_of_the_callers(M):
    """the inputs are written on the same stream just before, the results are read on it just after"""
    V, d = 900, 512
    w, h = rows_bf16(7, V, d, 0.02), rows_bf16(8, M, d)
    qw, sw = quantized(w)
    W, S, fresh = torch.from_numpy(qw).cuda(), torch.from_numpy(sw).cuda(), h.cuda()
    H, out = torch.zeros((M, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((M, V), device="cuda")
    ws, n = workspace(M, d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        busy = torch.zeros(1 << 28, device="cuda").add_(1).add_(1)
        H.copy_(fresh)
    B.nanospec_dense_head_i8(W, S, H, V, d, M, out, ws, n, stream=side)
    with torch.cuda.stream(side):
        copy = out.clone()
    side.synchronize()
    assert same(copy.cpu().numpy(), expected(qw, sw, *quantized(h))) and busy[0] == 2


@pytest.mark.parametrize("M", [1, 8, 16, 17, 64, 200])
def test_the_largest_sums_are_exact(M):
    V, d = 20, 133136
    qw = np.full((V, d), 127, np.int8)
    qw[::2] = -127
    qw[1, ::2] = -127
    sw = np.linspace(0.5, 2, V).astype(np.float32)
    h = torch.full((M, d), 3.0, dtype=torch.bfloat16)
    qh, sh = quantized(h)
    out = torch.empty((M, V), device="cuda")
    ws, n = workspace(M, d)
    B.nanospec_dense_head_i8(torch.from_numpy(qw).cuda(), torch.from_numpy(sw).cuda(), h.cuda(), V, d, M, out, ws, n)
    assert same(out.cpu().numpy(), expected(qw, sw, qh, sh))


def active_state(V, d, counts, M, cap=None):
    """a state whose sequence b holds counts[b] ids, and those ids"""
    top = cap or max(max(counts), 1)
    st = B.State(V, d, len(counts), 1, top, M, 1)
    ids = [np.sort(synth.rand_u64(40 + b, 0, 0, V).argsort()[:n]).astype(np.int32) for b, n in enumerate(counts)]
    off = np.zeros(len(counts) + 1, np.int32)
    off[1:] = np.cumsum(counts)
    flat = torch.from_numpy(np.concatenate(ids)).cuda() if off[-1] else None
    B.nanospec_vocab_init(st.h, None, np.zeros(len(counts) + 1, np.int32), flat, off)
    return st, ids


@pytest.mark.parametrize("counts,cap", [([1], None), ([0], 100), ([347], None), ([63, 0, 129], None), ([500] * 9, None), ([100], 3000), ([2500], None), ([700, 699, 0, 1], 900)])
@pytest.mark.parametrize("M,d", [(1, 512), (4, 48), (8, 4096), (16, 1040), (17, 512), (64, 256), (70, 2048)])
def test_active_rows_to_the_last_bit(counts, cap, M, d):
    V = 4001
    st, ids = active_state(V, d, counts, M, cap)
    w, h = rows_bf16(3, V, d, 0.02), rows_bf16(4, len(counts) * M, d)
    w[7] = 0
    (qw, sw), (qh, sh) = quantized(w), quantized(h)
    out = torch.full((len(counts), M, st.capacity), 5.0, device="cuda")
    ws, n = workspace(len(counts) * M, d)
    B.nanospec_sparse_head_i8(st.h, torch.from_numpy(qw).cuda(), torch.from_numpy(sw).cuda(), h.cuda(), M, out, ws, n)
    got = out.cpu().numpy()
    for b, live in enumerate(ids):
        k = len(live)
        if k:
            assert same(got[b, :, :k], expected(qw[live], sw[live], qh[b * M:(b + 1) * M], sh[b * M:(b + 1) * M])), b
        assert (got[b, :, k:] == 5.0).all(), b
    st.close()


def test_rows_whose_weights_are_not_finite_are_nan_and_no_others():
    V, d, M = 200, 512, 5
    w, h = rows_bf16(5, V, d, 0.02), rows_bf16(6, M, d)
    w[11, 3], w[199, 0] = float("inf"), float("nan")
    q, s = torch.empty((V, d), dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    B.nanospec_quantize_rows(w.cuda(), V, d, q, s)
    out = torch.empty((M, V), device="cuda")
    ws, n = workspace(M, d)
    B.nanospec_dense_head_i8(q, s, h.cuda(), V, d, M, out, ws, n)
    bad = torch.isnan(out).cpu().numpy()
    assert bad[:, [11, 199]].all() and bad.sum() == 2 * M


@pytest.mark.parametrize("M", [1, 4, 8, 20, 160])
def test_captured_and_replayed_on_another_stream(M):
    """two graphs with workspaces of their own, replayed in turn with eager work between; every replay is checked"""
    V, d = 700, 1024
    w, h = rows_bf16(7, V, d, 0.02), [rows_bf16(8 + i, M, d) for i in range(2)]
    qw, sw = quantized(w)
    W, S = torch.from_numpy(qw).cuda(), torch.from_numpy(sw).cuda()
    H = [x.cuda() for x in h]
    out = [torch.empty((M, V), device="cuda") for _ in range(2)]
    spaces = [workspace(M, d) for _ in range(2)]
    side = torch.cuda.Stream()
    graphs = []
    for i in range(2):
        B.nanospec_dense_head_i8(W, S, H[i], V, d, M, out[i], *spaces[i])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            B.nanospec_dense_head_i8(W, S, H[i], V, d, M, out[i], *spaces[i])
        graphs.append(g)
    for turn in range(3):
        fresh = [rows_bf16(50 + 2 * turn + i, M, d) for i in range(2)]
        for i in range(2):
            H[i].copy_(fresh[i])
            out[i].fill_(1.0)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert same(out[i].cpu().numpy(), expected(qw, sw, *quantized(fresh[i]))), (turn, i)


def test_refusals():
    V, d, M = 64, 64, 2
    L = B.lib()
    t = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda")
    W, S, H, out, ws = t(V * d + 16), t(4 * V), t(2 * M * d + 16), t(4 * M * V), t(4096)
    n = B.nanospec_head_i8_workspace(M, d)
    p = lambda x, o=0: C.c_void_p(x.data_ptr() + o)
    ok = dict(W=p(W), S=p(S), H=p(H), V=V, d=d, M=M, out=p(out), ws=p(ws), n=n)

    def dense(**k):
        a = {**ok, **k}
        return L.nanospec_dense_head_i8(a["W"], a["S"], a["H"], a["V"], a["d"], a["M"], a["out"], a["ws"], a["n"], None)

    assert dense() == B.OK
    for k in (dict(W=None), dict(S=None), dict(H=None), dict(out=None), dict(ws=None), dict(V=0), dict(M=0), dict(d=8), dict(d=24), dict(d=0), dict(d=133152), dict(W=p(W, 8)), dict(H=p(H, 2)),
              dict(ws=p(ws, 16)), dict(V=2 ** 31 - 1), dict(M=2 ** 31 - 1)):
        assert dense(**k) == B.EINVAL, k
    assert dense(n=n - 1) == B.ECAPACITY
    assert B.nanospec_head_i8_workspace(0, 64) == -1 and B.nanospec_head_i8_workspace(4, 40) == -1 and B.nanospec_head_i8_workspace(2 ** 31 - 1, 64) == -1
    assert L.nanospec_quantize_rows(None, 1, 16, p(W), p(S), None) == B.EINVAL
    assert L.nanospec_quantize_rows(p(H), 0, 16, p(W), p(S), None) == B.EINVAL
    assert L.nanospec_quantize_rows(p(H), 1, 20, p(W), p(S), None) == B.EINVAL
    assert L.nanospec_quantize_rows(p(H, 2), 1, 16, p(W), p(S), None) == B.EINVAL
    assert L.nanospec_quantize_rows(p(H), 2 ** 40, 16, p(W), p(S), None) == B.EINVAL
    st = B.State(V, d, 2, 4, 8, M, 1)
    sparse = lambda h, M_, n_: L.nanospec_sparse_head_i8(h, p(W), p(S), p(H), M_, p(out), p(ws), n_, None)
    assert sparse(None, 1, 4096) == B.EINVAL and sparse(st.h, 0, 4096) == B.EINVAL and sparse(st.h, M + 1, 4096) == B.ECAPACITY
    assert sparse(st.h, 1, B.nanospec_head_i8_workspace(2, d) - 1) == B.ECAPACITY
    odd = B.State(V, 24, 1, 4, 8, M, 1)                    # a state may have d % 8 == 0
    assert sparse(odd.h, 1, 4096) == B.EINVAL
    torch.cuda.synchronize()
