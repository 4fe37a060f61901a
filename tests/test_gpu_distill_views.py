"""Gradients whose rows are aligned otherwise than the logits', calls captured into a graph, and calls of several threads at
once: the same bits."""
import threading

import pytest
import torch

from paper_2506_01084_b200 import binding as zb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(dt, N, cols, K=9):
    g = torch.Generator(device=DEV)
    g.manual_seed(N + cols)
    n = (cols - torch.randint(0, cols // 3, (N,), generator=g, device=DEV)).int()
    n[0], n[1] = cols, 0
    ids = torch.randint(0, cols, (N, K), generator=g, device=DEV).int()
    ids[2] = -1
    w = torch.rand(N, generator=g, device=DEV) + 0.1
    w[N - 1] = 0.0
    w[N - 2] = -0.5
    return (torch.randn(N, cols, generator=g, device=DEV) * 2).to(dt), (n, ids, torch.randn(N, K, generator=g, device=DEV), 1.25), w


# rows held in shared memory by one and by several blocks, rows too long for that, the persistent form with clusters of one to
# eight; rows that are whole chunks of the ring and such that are not
FORMS = [(5, 1003), (4, 33001), (3, 1000003), (296, 70003), (80, 131072), (80, 262144), (75, 290001)]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,cols", FORMS)
@pytest.mark.parametrize("off_l,off_g", [(0, 1), (0, 3), (1, 0), (3, 2), (5, 5)])
def test_gradients_aligned_otherwise_than_the_logits(dt, N, cols, off_l, off_g):
    l, args, w = inputs(dt, N, cols)
    ld = cols + 16 - cols % 8
    buf = torch.full((N * ld + 8,), 777.0, dtype=dt, device=DEV)
    at = buf[off_l:].as_strided((N, cols), (ld, 1))
    at.copy_(l)
    want = buf.clone()[off_l:].as_strided((N, cols), (ld, 1))             # in place: aligned alike
    out = torch.empty(4, N, device=DEV)
    zb.z2z_distill_loss(want, *args, w, out[0], out[1], want)
    for backward in (False, True):
        g = torch.full((N * ld + 8,), 9.0, dtype=dt, device=DEV)
        view = g[off_g:].as_strided((N, cols), (ld, 1))
        if backward:
            zb.z2z_distill_grad(at, *args, out[1], w, view)
        else:
            zb.z2z_distill_loss(at, *args, w, out[2], out[3], view)
            assert torch.equal(out[:2], out[2:])
        assert torch.equal(view, want)
        view.fill_(9.0)
        assert (g == 9.0).all()
    assert torch.equal(at, l)


@pytest.mark.parametrize("N,cols", [(296, 70003), (80, 262144), (75, 290001)])
def test_the_persistent_form_replayed_from_a_graph(N, cols):
    l, args, w = inputs(torch.float32, N, cols)
    out = torch.empty(4, N, device=DEV)
    g = torch.empty(4, N, cols, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        zb.z2z_distill_loss(l, *args, w, out[0], out[1], g[0])
        zb.z2z_distill_grad(l, *args, out[1], w, g[1])
    for k in range(2):
        l.normal_()
        graph.replay()
        zb.z2z_distill_loss(l, *args, w, out[2], out[3], g[2])
        zb.z2z_distill_grad(l, *args, out[3], w, g[3])
        assert torch.equal(out[:2], out[2:]) and torch.equal(g[:2], g[2:])


def test_calls_of_several_threads_at_once():
    jobs = [inputs(dt, N, cols) for dt in (torch.bfloat16, torch.float32) for N, cols in ((76, 300007), (81, 580003), (7, 33001))]

    def run(l, args, w):
        out, g = torch.empty(2, l.shape[0], device=DEV), torch.empty_like(l)
        zb.z2z_distill_loss(l, *args, w, out[0], out[1], g)
        return out, g

    want = [run(*j) for j in jobs]
    torch.cuda.synchronize()
    got, start = [None] * len(jobs), threading.Barrier(len(jobs))

    def thread(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            start.wait(timeout=30)
            got[k] = [run(*jobs[k]) for _ in range(3)]
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=thread, args=(k,)) for k in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=60)
    for a, many in zip(want, got):
        assert all(torch.equal(x, y) for b in many for x, y in zip(a, b))
