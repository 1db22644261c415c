"""Orthogonalised updates: how near their products are to fp32's, by every kind of kernel, and momentum that is not kept.

Bounds.  An error made in a step grows through the later steps as any other one does, whatever products made it: against fp32 products on the same
input only what a step adds counts.  fp32 rounds what it stores by 0.4 2^-24 of it (root mean square) and its sums by about as much again;
two halves of 11 bits leave 0.24 2^-22 of a number, lo lo as much of a product, and their sums are fp32 too: together below 3 times
fp32's.  ALLOWED is twice that, of the largest error among some inputs, and 2^-21 where both are small.  One of the three products
lost leaves 2^-12 and more (tests/test_oracle_teaching_ends.py), a hundred times as much."""
import ctypes

import numpy as np
import pytest

from oracle import teaching as ot
from tests.test_gpu_losses import U, _host
from tests.test_gpu_orthogonal import USUAL, _mat, _round, bound, near

pytestmark = pytest.mark.gpu


def allowed(of_fp32):
    """Largest error of a factor, relative to its norm, where fp32 products have this one."""
    return 6.0 * of_fp32 + 2.0 ** -21


def _factor(x, mm):
    for a, b, c in USUAL:
        y = mm(x, x.T)
        x = a * x + mm(b * y + c * mm(y, y), x)
    return x


def _compare(grads, outs):
    """Errors of fp32 products and of the outputs, relative to the factors' norms."""
    import torch
    for g, out in zip(grads, outs):
        x, got = (g.double(), out.double()) if g.shape[0] <= g.shape[1] else (g.double().T.contiguous(), out.double().T)
        x = x / (x.norm() + 1e-7)
        exact, fp32 = _factor(x, lambda p, q: torch.mm(p, q.contiguous())), _factor(x.float(), lambda p, q: torch.mm(p, q.contiguous()))
        yield tuple(float((f.double() - exact).norm() / exact.norm()) for f in (fp32, got))


# a workgroup each (up to 16, 32 and 64 rows, of 128 to 4096), in tiles of every kind, with shared sums, eight in turns, tall and wide
SHAPES = [([(1, 7)], 12), ([(5, 94)], 12), ([(51, 7)], 12), ([(16, 211)], 12), ([(16, 500)], 12), ([(16, 1000)], 12), ([(16, 2000)], 12), ([(4000, 16)], 12),
          ([(17, 100)], 12), ([(31, 500)], 12), ([(32, 1000)], 12), ([(32, 2000)], 12), ([(64, 64)], 12), ([(500, 60)], 12), ([(64, 1000)], 12),
          ([(16, 211)] * 9 + [(60, 700)] * 9 + [(20, 1500)] * 9 + [(10, 3000)] * 3, 2), ([(65, 65)], 6), ([(130, 70)], 6), ([(128, 4096)], 3), ([(333, 1111)], 3), ([(1111, 333)] * 3 + [(257, 1001)] * 2, 3), ([(70, 30001)], 3), ([(512, 512)] * 9, 2),
          ([(1024, 1024)], 2), ([(1536, 1600)] * 8, 1), ([(2001, 1999)], 2), ([(2500, 2600)], 1), ([(1024, 4096)] * 4, 1), ([(4096, 4100)], 1), ([(8000, 4096)], 1)]


@pytest.mark.parametrize("shapes,draws", SHAPES)
def test_products_are_as_near_as_those_of_fp32(shapes, draws):
    import torch
    import paper_1906_08879_amd as pl
    gen = torch.Generator("cuda").manual_seed(len(shapes) + shapes[0][0])
    worst = {}
    for _ in range(draws):
        grads = [torch.randn(s, device="cuda:0", generator=gen) for s in shapes]
        outs = [torch.empty_like(g) for g in grads]
        pl.orthogonal_update(grads, out=outs)
        for s, (fp32, got) in zip(shapes, _compare(grads, outs)):
            worst[s] = tuple(max(p) for p in zip(worst.get(s, (0.0, 0.0)), (fp32, got)))
    for s, (fp32, got) in worst.items():
        print(f"[orthogonal] {s}: {got:.2e}, by fp32 products {fp32:.2e}", flush=True)
        assert got <= allowed(fp32), (s, got, fp32)


FEW = [(1, 1), (1, 7), (3, 2), (16, 16), (15, 33), (17, 17), (32, 32), (31, 97), (100, 29), (5, 3001), (16, 4095), (4096, 16), (30, 2047), (2048, 32),
       (16, 4097), (5000, 9), (2, 20001), (32, 2049), (2049, 17), (29, 30001), (1, 300001)]


@pytest.mark.parametrize("shape", FEW)
def test_few_rows_lose_nothing(shape):
    """Up to 32 rows everything is float64: the results have their last rounding alone, 2^-24 of an element, and what the products of float64 leave,
    below 1e-9.  All together, then with 32 steps, other factors, and of low rank."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(shape[0] + shape[1])
    k = min(shape)
    g = rng.normal(0, 1, shape)
    low = rng.normal(0, 1, (shape[0], max(1, k // 2))) @ rng.normal(0, 1, (max(1, k // 2), shape[1]))
    for a, iteration in ((g, USUAL), (low, USUAL), (g * np.logspace(0, -5, shape[1]), USUAL), (g, ((1.5, -0.5, 0.0),) * 32), (g, ((1.0, 0.0, 0.0),)),
                         (g, ((2.0, -1.5, 0.5),) * 9), (1e-30 * g, ((8.0, -20.0, 15.0), (3.0, -3.0, 1.0)))):
        a = _round(a, "fp32")
        steps = [tuple(float(np.float32(v)) for v in step) for step in iteration]
        out = _mat(np.full(shape, 7.0), "fp32", 1, 1)
        pl.orthogonal_update([_mat(a, "fp32", 3, 1)], out=[out], iteration=iteration, eps=0.0)
        x = a if shape[0] >= shape[1] else a.T            # (the oracle's products are those of the columns)
        x, _, _ = ot.orthogonal(x, iteration=steps, eps=0.0)
        x = x if shape[0] >= shape[1] else x.T
        assert np.linalg.norm(_host(out) - x) <= (2.0 ** -24 + 1e-9) * np.linalg.norm(x), (shape, iteration)


def test_many_of_few_rows_through_lists():
    """More than go by value, those of a workgroup each and those in parts; in place, with momentum."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(3)
    shapes = [s for s in FEW if max(s) < 40000] * 3 + [(3, 5000 + 700 * i) for i in range(25)] + [(40, 50), (70, 80)]
    host = [_round(rng.normal(0, 1, s), "bf16") for s in shapes]
    grads, moments = [_mat(h, "bf16", 1, 1) for h in host], [_mat(np.zeros(s), "fp32", 2) for s in shapes]
    weights = [torch.ones(s, device="cuda:0") for s in shapes]
    pl.orthogonal_update(grads, moments, weights=weights, out=grads, lr=0.5, nesterov=False)
    for h, g, m, w in zip(host, grads, moments, weights):
        wide = h.shape[0] < h.shape[1]
        x, _, xs = ot.orthogonal(h.T if wide else h)
        x = x.T if wide else x
        tol = bound(xs, USUAL, 4.0) if min(h.shape) > 32 else 2.0 ** -22 * np.linalg.norm(x)        # (factors of fp32)
        assert np.array_equal(_host(m), h)
        near(_host(g), x, tol, "bf16")
        near(_host(w), 1.0 - 0.5 * x, 0.5 * tol + 4 * U * np.sqrt(x.size), "fp32")


@pytest.mark.parametrize("shapes", [[(16, 5000), (9000, 3), (20, 30001)], [(5, 5000)] * 30 + [(30, 3000), (64, 64)]])
def test_replays_of_long_matrices_of_few_rows(shapes):
    import torch
    import paper_1906_08879_amd as pl
    grads, m, w = ([torch.randn(s, device="cuda:0") for s in shapes] for _ in range(3))
    om, ow, out = ([torch.empty(s, device="cuda:0") for s in shapes] for _ in range(3))
    ws = torch.empty(pl.orthogonal_workspace_bytes(shapes), dtype=torch.uint8, device="cuda:0")

    def call():
        pl.orthogonal_update(grads, m, om, w, ow, out, scales=0.5, decay=0.1, workspace=ws)

    call()
    torch.cuda.synchronize()
    outs = om + ow + out
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        for t in outs:
            t.fill_(3 + i)
        ws.fill_(255 - i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, u) for t, u in zip(outs, want)), i
        call()
        torch.cuda.synchronize()


@pytest.mark.parametrize("shape", [(7, 90), (16, 4096), (90, 30), (20, 5000), (5000, 3)])
def test_norms_of_few_rows_at_the_ends(shape):
    """Nothing but zeros stays zero; one element that is no number makes the matrix none, and no other one."""
    import torch
    import paper_1906_08879_amd as pl
    zero, out = torch.zeros(shape, device="cuda:0"), torch.full(shape, 7.0, device="cuda:0")
    for eps in (0.0, 1e-7):
        pl.orthogonal_update([zero], out=[out.fill_(7.0)], eps=eps)
        assert (out == 0).all()
    for bad in (float("nan"), float("inf"), -float("inf")):
        h, other, oo = torch.zeros(shape, device="cuda:0"), torch.randn((9, 9), device="cuda:0"), torch.empty((9, 9), device="cuda:0")
        h[-1, -2] = bad
        pl.orthogonal_update([h, other], out=[out.zero_(), oo])
        assert torch.isnan(out).all() and torch.isfinite(oo).all()
    for s in (1e37, 1e-40):
        g = _round(np.random.default_rng(1).normal(0, 1, shape) * s, "fp32")
        x = g if shape[0] >= shape[1] else g.T
        x, _, _ = ot.orthogonal(x, iteration=[tuple(float(np.float32(v)) for v in step) for step in USUAL], eps=0.0)
        pl.orthogonal_update([_mat(g, "fp32")], out=[out], eps=0.0)
        x = x if shape[0] >= shape[1] else x.T
        assert np.linalg.norm(_host(out) - x) <= (2.0 ** -24 + 1e-9) * np.linalg.norm(x)


@pytest.mark.parametrize("rows,cols,rank", [(15, 200, 10), (60, 40, 30), (200, 150, 120), (700, 1300, 200)])
def test_products_of_nearly_low_rank(rows, cols, rank):
    """Singular values over six orders: the smallest, and errors with them, grow most."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(rows)
    worst = [0.0, 0.0]
    for _ in range(4):
        q, r = (np.linalg.qr(rng.normal(0, 1, (n, rank)))[0] for n in (rows, cols))
        g = _mat((q * np.logspace(0, -6, rank)) @ r.T, "fp32")
        out = torch.empty(g.shape, device="cuda:0")
        pl.orthogonal_update([g], out=[out])
        worst = [max(p) for p in zip(worst, *_compare([g], [out]))]
    print(f"[orthogonal] {rows} x {cols} of rank {rank}: {worst[1]:.2e}, by fp32 products {worst[0]:.2e}", flush=True)
    assert worst[1] <= allowed(worst[0]), worst


@pytest.mark.parametrize("nesterov", [0, 1])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 4), (40, 70), (60, 64), (3000, 16), (20, 9000), (9000, 5), (300, 129), (70, 3000)])
def test_momentum_that_is_not_kept(shape, dtype, nesterov):
    """new_momentum NULL, of one matrix beside another whose momentum is kept: the direction is that of the new momentum, the old one stays."""
    import torch
    import paper_1906_08879_amd as pl
    from paper_1906_08879_amd import binding as b
    rng = np.random.default_rng(shape[1] + nesterov)
    g, m, w = (_round(rng.normal(0, s, shape), d) for s, d in ((1e-2, dtype), (3e-2, "fp32"), (0.3, dtype)))
    code = {"fp32": 0, "bf16": 1}[dtype]
    tg, views, kept = _mat(g, dtype, 1, 1), (b.MatrixView * 2)(), []
    for i in range(2):
        tm, tw, out, new = _mat(m, "fp32", 2), _mat(w, dtype, 3), torch.empty(shape, device="cuda:0"), torch.full(shape, 7.0, device="cuda:0")
        kept.append((tm, tw, out, new))
        views[i] = b.MatrixView(*shape, code, code, 0, 1.7, tg.data_ptr(), tg.stride(0), tm.data_ptr(), tm.stride(0), new.data_ptr() if i else None,
                                new.stride(0) if i else 0, tw.data_ptr(), tw.stride(0), tw.data_ptr(), tw.stride(0), out.data_ptr(), out.stride(0))
    factors = (ctypes.c_float * 15)(*[f for step in USUAL for f in step])
    cfg = b.OrthogonalCfg(0.3, 0.1, 0.9, 1e-7, nesterov, 5, ctypes.cast(factors, ctypes.c_void_p))
    lib = pl.load_library()
    ws = torch.empty(lib.pl_orthogonal_workspace(2, views), dtype=torch.uint8, device="cuda:0")
    assert lib.pl_orthogonal_update(2, views, ctypes.byref(cfg), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    x, new_m, xs = ot.orthogonal(g, m, 0.9, bool(nesterov))
    want = (1.0 - 0.3 * 0.1) * w - 0.3 * 1.7 * x
    # the direction in fp32: two roundings of its terms, over its norm
    d = 4 * U * (np.linalg.norm(g) + np.linalg.norm(new_m) + np.linalg.norm(m)) / np.linalg.norm(g + 0.9 * new_m if nesterov else new_m) * 4.0 ** 5
    tol = bound(xs, USUAL, 4.0) + d
    for i, (tm, tw, out, new) in enumerate(kept):
        assert np.array_equal(_host(tm), m)
        near(_host(out), x, tol, "fp32")
        near(_host(tw), want, 0.3 * 1.7 * tol + 8 * U * np.linalg.norm(w), dtype)
        assert (new == 7).all() if not i else (np.abs(_host(new) - new_m) <= 2 * U * (np.abs(new_m) + 0.9 * np.abs(m))).all()
    d = _host(kept[0][2]) - _host(kept[1][2])             # both ways to the direction: its roundings alone
    assert np.linalg.norm(d) <= 2 * 4 * U * 4.0 ** 5 * np.linalg.norm(x)
