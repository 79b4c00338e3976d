"""What the launch trace says of token launches over tenants of several sizes: the operations of all of them."""
import pytest
import torch  # before the library: both then share one HIP runtime

from test_gpu_tokens import Pick, Tenant, decode, draw, feature, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", [([(5, 300), (60, 7001), (0, 999)], 128, False), ([(400, 300), (31, 7001), (0, 5)], 128, False),
                                  ([(400, 300), (31, 7001), (100, 64)], 256, True), ([(30, 60001), (7, 40001)], 256, True),
                                  ([(2000, 300007), (31, 70)], 64, True), ([(3 + k, 200 + 90 * k) for k in range(30)], 128, False)],
                         ids=lambda c: "")
def test_operations_of_a_call(lib, case):
    sizes, d, dh = case
    hidden = feature(500, d)
    ts = [Tenant(lib, *draw(n, v, d, 500, 120 + k), dh) for k, (n, v) in enumerate(sizes)]
    ctx = lib.Context()
    ctx.set_trace(True)
    step(lib, ctx, hidden, ts)
    trace = ctx.trace_read()
    products = [(M, N, K) for op, M, N, K, _ in trace if op == "token_gemm"]
    once = sum(n * v * d for n, v in sizes)
    # columns behind the kept piece are formed twice, and few rows' dh takes two rows an entry
    assert 0 < min(M * N * K for M, N, K in products)
    total, rounding = sum(M * N * K for M, N, K in products), sum(max(M * N, M * K, N * K) for M, N, K in products)
    assert (3 if dh else 2) * once - rounding <= total <= (4 if dh else 2) * once + rounding
    rows = [N for op, M, N, K, _ in trace if op == "token_other" and N not in (d,)]
    assert all(min(v for n, v in sizes if n) <= N <= max(v for n, v in sizes if n) for N in rows)
    picks = [Pick(lib, t.W, t.rows) for t in ts]
    ctx.set_trace(True)
    decode(lib, ctx, hidden, picks)
    products = [(M, N, K) for op, M, N, K, _ in ctx.trace_read() if op == "token_gemm"]
    total, rounding = sum(M * N * K for M, N, K in products), sum(M * K for M, N, K in products)
    assert abs(total - once) <= rounding
