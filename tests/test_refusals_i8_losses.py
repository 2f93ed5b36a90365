"""What the 8-bit heads and the losses refuse, found on the host before anything is launched: no GPU, addresses that are never read."""
import ctypes as C
import os

import numpy as np
import pytest

import choose
import choose_i8
from paper_2605_26444_amd import binding as B

P = 1 << 20                                                # an address, aligned to everything


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2605_26444_amd import build
        build.build()
    return B.lib()


def test_workspaces():
    assert B.nanospec_head_i8_workspace(8, 4096) >= 8 * 4096 + 8 * 4
    for rows, d in ((0, 64), (-1, 64), (4, 0), (4, 8), (4, 40), (4, 133152), (2 ** 31 - 1, 64)):
        assert B.nanospec_head_i8_workspace(rows, d) == -1, (rows, d)
    assert B.nanospec_head_i8_workspace(2 ** 24 + 1, 16) == -1 and B.nanospec_head_i8_workspace(2 ** 24, 16) > 0
    for rows, V in ((0, 5), (5, 0), (-3, 5), (5, 2 ** 30 + 1), (2 ** 22 + 1, 1), (2 ** 31 - 1, 1)):
        assert B.nanospec_loss_workspace(rows, V) == -1, (rows, V)
    sizes = [(1, 1), (7, 32000), (509, 128256), (2048, 152064), (2 ** 22, 1), (3, 2 ** 30)]
    assert all(B.nanospec_loss_workspace(r, v) >= 24 * r for r, v in sizes)


@pytest.mark.parametrize("change", [dict(W=None), dict(S=None), dict(H=None), dict(out=None), dict(ws=None), dict(V=0), dict(V=-1), dict(M=0), dict(d=0), dict(d=8), dict(d=24),
                                    dict(d=133152), dict(W=P + 8), dict(H=P + 2), dict(ws=P + 16), dict(V=2 ** 31 - 1), dict(M=2 ** 31 - 1), dict(M=2 ** 24 + 1)])
def test_dense_head_i8(lib, change):
    a = {**dict(W=P, S=P, H=P, V=64, d=64, M=2, out=P, ws=P, n=1 << 40), **change}
    assert lib.nanospec_dense_head_i8(a["W"], a["S"], a["H"], a["V"], a["d"], a["M"], a["out"], a["ws"], a["n"], None) == B.EINVAL


def test_workspace_too_small_and_rows_to_quantize(lib):
    assert lib.nanospec_dense_head_i8(P, P, P, 64, 64, 2, P, P, B.nanospec_head_i8_workspace(2, 64) - 1, None) == B.ECAPACITY
    assert lib.nanospec_sparse_head_i8(None, P, P, P, 1, P, P, 1 << 40, None) == B.EINVAL
    for x, rows, d, q, s in ((None, 1, 16, P, P), (P, 1, 16, None, P), (P, 1, 16, P, None), (P, 0, 16, P, P), (P, 1, 20, P, P), (P + 2, 1, 16, P, P), (P, 1, 16, P + 8, P), (P, 2 ** 40, 16, P, P)):
        assert lib.nanospec_quantize_rows(x, rows, d, q, s, None) == B.EINVAL, (rows, d)


def source(**k):
    r = B.LogitRows(P, P, None, None, 64, B.F32, 4, 32, 1)
    for name, value in k.items():
        setattr(r, name, value)
    return r


def policy(lib, rows=None, **k):
    a = {**dict(old=P, ref=P, adv=P, w=None, lo=0.2, hi=0.2, kl=0.1, loss=P, grad=None, kind=B.F32, ld=32, scale=1.0, ws=P, n=1 << 40), **k}
    return lib.nanospec_policy_loss(rows if rows is not None else source(), a["old"], a["ref"], a["adv"], a["w"], a["lo"], a["hi"], a["kl"], a["loss"], None, None, a["grad"], a["kind"],
                                    a["ld"], a["scale"], a["ws"], a["n"], None)


def pair(lib, off, rows=None, pairs=None, **k):
    a = {**dict(ref=None, w=None, beta=0.1, e=0.0, loss=P, grad=None, kind=B.F32, ld=32, scale=1.0, ws=P, n=1 << 40), **k}
    o = None if off is None else np.asarray(off, np.int32)
    return lib.nanospec_preference_loss(rows if rows is not None else source(), None if o is None else o.ctypes.data, len(o) // 2 if pairs is None else pairs, a["ref"], a["w"], a["beta"],
                                        a["e"], a["loss"], None, None, a["grad"], a["kind"], a["ld"], a["scale"], a["ws"], a["n"], None)


@pytest.mark.parametrize("change", [dict(d_logits=None), dict(d_tokens=None), dict(rows=0), dict(rows=-1), dict(rows=2 ** 22 + 1), dict(V=0), dict(V=2 ** 30 + 1), dict(ld=31), dict(ld=2 ** 60), dict(type=2), dict(d_logits=P + 2),
                                    dict(type=-1), dict(d_ids=P), dict(d_n=P), dict(d_ids=P, d_n=P, rows_per_list=0)])
def test_rows_of_logits(lib, change):
    assert policy(lib, source(**change)) == B.EINVAL
    assert pair(lib, [0, 2, 4], source(**change)) == B.EINVAL
    assert lib.nanospec_token_logprob(source(**change), P, P, 1 << 40, None) == B.EINVAL


NAN = float("nan")


@pytest.mark.parametrize("change", [dict(old=None), dict(adv=None), dict(loss=None), dict(ref=None), dict(lo=-0.1), dict(hi=-1.0), dict(lo=NAN), dict(hi=NAN), dict(kl=NAN), dict(scale=NAN),
                                    dict(ws=None), dict(ws=P + 8), dict(grad=P + (1 << 20), kind=7), dict(grad=P + (1 << 20), ld=31), dict(grad=P + (1 << 20) + 2), dict(grad=P, kind=B.BF16, ld=64),
                                    dict(grad=P, ld=65), dict(grad=P + 4, ld=64), dict(grad=P + 4 * 64, ld=64), dict(grad=P - 4, ld=64)])
def test_policy_loss(lib, change):
    assert policy(lib, **change) == B.EINVAL


@pytest.mark.parametrize("change", [dict(beta=NAN), dict(e=-0.1), dict(e=1.1), dict(e=NAN), dict(loss=None), dict(ws=None), dict(grad=P, ld=65), dict(scale=NAN)])
def test_preference_loss(lib, change):
    assert pair(lib, [0, 2, 4], **change) == B.EINVAL


def test_offsets_of_answers(lib):
    for off in ([0, 3, 2], [-1, 2, 4], [0, 2, 5]):
        assert pair(lib, off) == B.EINVAL, off
    assert pair(lib, None, pairs=1) == B.EINVAL and pair(lib, [0, 2, 4], pairs=0) == B.EINVAL and pair(lib, [0, 2, 4], pairs=-1) == B.EINVAL
    assert pair(lib, [0] * 259) == B.ECAPACITY
    assert pair(lib, [0, 2, 4], n=B.nanospec_loss_workspace(4, 32) - 1) == B.ECAPACITY and policy(lib, n=B.nanospec_loss_workspace(4, 32) - 1) == B.ECAPACITY
    assert lib.nanospec_token_logprob(None, P, P, 1 << 40, None) == B.EINVAL and lib.nanospec_token_logprob(source(), None, P, 1 << 40, None) == B.EINVAL
    with pytest.raises(ValueError):
        B.nanospec_preference_loss(source(), [0, 2], None, None, 0.1, 0.0, P, None, None, None, P, 1 << 40)


@pytest.mark.parametrize("M", range(1, 17))
def test_shapes_of_the_few_row_head_fit_the_chip(M):
    for d in range(16, 16400, 16):
        if not choose_i8.few_supported(M, d):
            continue
        for batch, cap in ((1, 64), (1, 128256), (64, 2304), (5, 9024), (256, 64), (1, 1 << 27)):
            f = choose_i8.few_plan(M, d, batch, cap)
            assert 1 <= f.waves <= 8 and f.waves == f.slices << f.log_groups and 256 * f.KS * f.slices >= d and (f.KS < 8 or M <= 8)
            assert f.seg >= 4 and f.seg % 4 == 0 and f.seg * (4 << f.log_groups) <= 2 * 64 * f.waves       # two scales a thread
            mh = 4 if M <= 4 else 8 if M <= 8 else 16
            rows = f.seg * (4 << f.log_groups)
            held = M * (d + 16) if choose_i8.few_rounds(M, d) else 0
            assert f.lds == 64 + 4 * rows + max(held, 4 * f.slices * mh * (rows + 4)) <= 80 * 1024        # two workgroups a compute unit
            assert 0 <= f.log_parts <= 5


@pytest.mark.parametrize("M,d,batch,cap,want", [(8, 4096, 1, 3008, (2, 8)), (8, 4096, 1, 128256, (8, 4)), (1, 512, 1, 384, (2, 8)), (16, 4096, 1, 32768, (4, 4)), (8, 4096, 64, 2304, (8, 4)),
                                                (16, 8192, 1, 3008, (4, 8)), (8, 2048, 1, 128256, (4, 8)), (16, 512, 1, 128256, (2, 8))])
def test_shape_of_the_few_row_head(M, d, batch, cap, want):
    f = choose_i8.few_plan(M, d, batch, cap)
    assert (f.KS, f.waves) == want


@pytest.mark.parametrize("M,d,batch,cap,dense,want", [
    (32, 4096, 1, 3008, False, "32x32"), (32, 4096, 1, 9024, False, "64x32"), (64, 3584, 1, 3008, False, "32x32"), (60, 4096, 4, 2048, False, "32x64"), (64, 4096, 1, 9024, False, "64x64"),
    (256, 4096, 1, 8000, True, "128x64"), (64, 4096, 1, 128256, True, "64x64"), (60, 4096, 64, 2304, False, "128x64"), (100, 4096, 1, 50000, True, "256x128"),
    (200, 4096, 1, 30016, False, "256x128"), (256, 4096, 1, 50000, True, "gemm"), (1024, 4096, 1, 128256, True, "gemm"), (1024, 4112, 1, 128256, True, "256x128")])
def test_block_shape_of_the_8_bit_head(M, d, batch, cap, dense, want):
    assert choose.rows_by_hidden(choose_i8.i8_shape(M, d, batch, cap, dense)) == want


class Elsewhere:
    """stands for a tensor of another device"""

    def get_device(self):
        return 3


def test_tensors_of_another_device(lib, monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    e = Elsewhere()
    rows = source()
    rows.keep = (e,)
    for call in (lambda: B.nanospec_quantize_rows(e, 1, 16, P, P), lambda: B.nanospec_dense_head_i8(P, P, e, 64, 64, 1, P, P, 1 << 40),
                 lambda: B.nanospec_token_logprob(rows, P, P, 1 << 40), lambda: B.nanospec_policy_loss(source(), P, P, P, None, 0.2, 0.2, 0.1, e, None, None, None, P, 1 << 40),
                 lambda: B.nanospec_preference_loss(source(), [0, 1, 2], None, None, 0.1, 0.0, P, None, None, e, P, 1 << 40)):
        with pytest.raises(ValueError, match="device 3"):
            call()
