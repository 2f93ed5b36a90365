"""The 8-bit head over active sets in the forms between its kernels -- hidden rows rounded by a launch of their own in front of the few-row kernel, several
sequences on each block shape -- and captured: logits to the last bit, as test_gpu_head_i8.py asks for."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import test_gpu_head_i8 as T
from paper_2605_26444_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts,cap", [([347], None), ([63, 0, 129, 1], None), ([2500, 1], 3000)])
@pytest.mark.parametrize("M,d", [(16, 4096), (9, 4080), (3, 8192), (8, 8208), (2, 16384), (16, 8192), (12, 2736)])
def test_few_hidden_rows_rounded_before(counts, cap, M, d):
    T.test_active_rows_to_the_last_bit(counts, cap, M, d)


@pytest.mark.parametrize("counts", [[3900] * 2 + [0, 11], [3000] * 4, [1500] * 24])
@pytest.mark.parametrize("M", [18, 33, 64, 65, 100])
def test_several_sequences_on_every_block_shape(counts, M):
    T.test_active_rows_to_the_last_bit(counts, None, M, 272)


@pytest.mark.parametrize("M,d", [(4, 512), (16, 4096), (40, 1024)])
def test_captured_while_the_active_sets_change(M, d):
    """a draft step's head in a graph: the sets change between the replays, by calls outside of it"""
    V, batch = 3001, 3
    st = B.State(V, d, batch, 400, 900, M, 1)
    g = np.random.RandomState(M)
    start = [np.sort(g.permutation(V)[:n]).astype(np.int32) for n in (700, 5, 300)]
    off = np.array([0, 700, 705, 1005], np.int32)
    B.nanospec_vocab_init(st.h, None, np.zeros(batch + 1, np.int32), torch.from_numpy(np.concatenate(start)).cuda(), off)
    w, h = T.rows_bf16(3, V, d, 0.02), T.rows_bf16(4, batch * M, d)
    (qw, sw), (qh, sh) = T.quantized(w), T.quantized(h)
    W, S, H = torch.from_numpy(qw).cuda(), torch.from_numpy(sw).cuda(), h.cuda()
    out = torch.full((batch, M, st.capacity), 5.0, device="cuda")
    ws, n = T.workspace(batch * M, d)
    call = lambda: B.nanospec_sparse_head_i8(st.h, W, S, H, M, out, ws, n)
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call()
    for turn in range(4):
        if turn:
            fresh = torch.from_numpy(g.randint(0, V, 60 * batch).astype(np.int32)).cuda()
            B.nanospec_vocab_update(st.h, fresh, np.arange(0, 60 * batch + 1, 60).astype(np.int32))
        out.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        for b, live in enumerate(st.read_active()):
            k = len(live)
            assert T.same(got[b, :, :k], T.expected(qw[live], sw[live], qh[b * M:(b + 1) * M], sh[b * M:(b + 1) * M])), (turn, b)
            assert (got[b, :, k:] == 5.0).all(), (turn, b)
    st.close()
