"""Split products of several host threads on one stream: the partial sums' launch and the join of a call are
queued with no other call between, so every result has the bits of a call by itself."""
import threading

import numpy as np
import pytest

import synthdata
from oracle import q8
from test_gpu_q8 import env, operand  # noqa: F401

pytestmark = pytest.mark.gpu

CALLS = 150


def together(torch, *work):
    """Each of these CALLS times, a thread for each, started together."""
    start, errors = threading.Barrier(len(work)), []

    def loop(fn):
        try:
            start.wait()
            for i in range(CALLS):
                fn(i)
        except Exception as e:                         # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=loop, args=(fn,)) for fn in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors


def product(torch, L, rng, M, K, N, name):
    """(operands, outputs of all calls, what one call by itself gives), a shape that splits its reduction."""
    a, _ = operand(torch, L, rng, M, K, q8.E4M3, q8.POW2, 1)
    b, _ = operand(torch, L, rng, N, K, q8.E4M3, q8.POW2, 128)
    want = torch.empty(M, N, dtype=getattr(torch, name), device="cuda")
    L.ds_q8_matmul(a, b, want)
    torch.cuda.synchronize()
    return a, b, torch.empty(CALLS, M, N, dtype=want.dtype, device="cuda"), want


@pytest.mark.parametrize("own_streams", [False, True])
def test_products(env, own_streams):  # noqa: F811
    """On one stream that the threads share, and on the handle that is another stream in each thread."""
    torch, L = env
    rng = np.random.default_rng(43)
    cases = [product(torch, L, rng, *shape) for shape in
             ((40, 8192, 64, "bfloat16"), (33, 6000, 100, "float32"), (3, 8300, 300, "bfloat16"))]
    stream = 2 if own_streams else torch.cuda.Stream()     # hipStreamPerThread
    together(torch, *[lambda i, c=c: L.ds_q8_matmul(c[0], c[1], c[2][i], stream=stream) for c in cases])
    for _, _, got, want in cases:
        assert all(torch.equal(got[i], want) for i in range(CALLS))


def test_threads_one_after_another(env):  # noqa: F811
    """Threads that end with work on their way, each on its own stream of one handle: a later thread may have an
    earlier one's id."""
    torch, L = env
    rng = np.random.default_rng(59)
    cases = [product(torch, L, rng, *shape) for shape in ((200, 8192, 900, "float32"), (40, 8192, 64, "float32"))]

    def once(i):
        a, b, got, _ = cases[i % 2]
        L.ds_q8_matmul(a, b, got[i], stream=2)

    for i in range(40):
        t = threading.Thread(target=once, args=(i,))
        t.start()
        t.join()
    torch.cuda.synchronize()
    assert all(torch.equal(cases[i % 2][2][i], cases[i % 2][3]) for i in range(40))


def test_beside_a_split_schedule(env):  # noqa: F811
    """kernel_run's split schedules use the same workspace."""
    torch, L = env
    rng = np.random.default_rng(47)
    sh = (1, 64, 40, 40, 64, 3, 3, 1, 1)
    x, w = (torch.from_numpy(v).cuda() for v in synthdata.conv_inputs(sh, "uniform"))
    s = L.Space(L.DS_OP_CONV2D_NCHW, sh).sched_of(tk=16, th=4, tw=32, tc=16, unroll=0, lds=1, ks=4, mfma=1, vec=4)
    alone = torch.empty(64 * 40 * 40, device="cuda")
    L.kernel_run(L.DS_OP_CONV2D_NCHW, s, x, w, alone)
    conv = torch.empty(CALLS, alone.numel(), device="cuda")
    a, b, got, want = product(torch, L, rng, 40, 8192, 64, "float32")
    st = torch.cuda.Stream()
    together(torch, lambda i: L.ds_q8_matmul(a, b, got[i], stream=st),
             lambda i: L.kernel_run(L.DS_OP_CONV2D_NCHW, s, x, w, conv[i], st))
    assert all(torch.equal(got[i], want) and torch.equal(conv[i], alone) for i in range(CALLS))
