"""The grouped products as a program uses them: experts put together from them, training steps, 8-bit experts, captured graphs,
streams, shared workspaces, buffers beyond 32 bits; and shapes for every way in which their kernels cut a call.

Tolerances as in test_gpu_products.py; where operators follow one another they are carried through the formulas, see each test.
u below is fp32's half step 2^-24, h bf16's 2^-8."""
import math

import pytest
import torch

from paper_2501_10375_amd import moe, products
from test_gpu_products import BF16, DEV, F32, UNTOUCHED, check, normal, quantised, reference, same_bits, table, workspace

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -8
SILU_SLOPE, SILU_BEND = 1.1, 0.5   # bounds of silu' (1.0998) and of |silu''| (0.5)


def selections(T, E, k, hidden, seed=0):
    """Routed tokens: x, the rows of x in the experts' order, offsets, and which selection each row is."""
    shape = moe.make_shape(hidden, 64, E, k, BF16)
    x, gate = normal(T, hidden, dtype=BF16, seed=seed + 1), normal(E, hidden, dtype=BF16, seed=seed + 2, std=0.05)
    idx, w = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    counts = torch.empty(E, dtype=torch.int32, device=DEV)
    moe.moe_route(shape, x, gate, None, idx, w, counts, False, moe.alloc_workspace(shape, T))
    order = torch.argsort(idx.flatten(), stable=True)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device=DEV)
    offsets[1:] = counts.cumsum(0)
    return x, idx, w, order, offsets


@pytest.mark.parametrize("T,E,k,hidden,ffn", [(1, 8, 2, 256, 512), (33, 8, 2, 512, 704), (300, 16, 4, 320, 576)])
def test_experts_of_products_are_the_fused_experts(T, E, k, hidden, ffn):
    """moe_route, three products and a sum against moe_expert_ffn.  g and u are rounded to bf16 here (h of each), so silu(g) u is off by
    at most h (1.1 |g| |u| + |silu(g)| |u|), and both round it and the sum over the selections; here the third product's
    result is rounded too.  Carried through |w2| and the selections' weights; 4 % for terms of second order, and the fp32 sums."""
    x, idx, topk_w, order, offsets = selections(T, E, k, hidden)
    w1, w3, w2 = (normal(E, *s, dtype=BF16, seed=7 + i, std=0.06) for i, s in enumerate(((ffn, hidden), (ffn, hidden), (hidden, ffn))))
    R = T * k
    rows = x[order // k].contiguous()
    ws = workspace(E, ffn, hidden, BF16, R)
    g, u, out = (torch.empty(R, n, dtype=BF16, device=DEV) for n in (ffn, ffn, hidden))
    products.moe_grouped_product(rows, offsets, w1, g, ws)
    products.moe_grouped_product(rows, offsets, w3, u, ws)
    act = (torch.nn.functional.silu(g.float()) * u.float()).to(BF16)
    products.moe_grouped_product(act, offsets, w2, out, ws)
    weight = topk_w.flatten()[order]
    y = torch.zeros(T, hidden, dtype=torch.float64, device=DEV).index_add_(0, order // k, out.double() * weight.double()[:, None])

    fused = torch.empty(T, hidden, dtype=BF16, device=DEV)
    shape = moe.make_shape(hidden, ffn, E, k, BF16)
    moe.moe_expert_ffn(shape, x, idx, topk_w, w1, w3, w2, fused, moe.alloc_workspace(shape, T))

    o = offsets.tolist()
    bound = torch.zeros(T, hidden, dtype=torch.float64, device=DEV)
    value = torch.zeros_like(bound)
    for e in range(E):
        r = slice(o[e], o[e + 1])
        gd, ud = rows[r].double() @ w1[e].double().T, rows[r].double() @ w3[e].double().T
        sums = (hidden + 8) * U * (rows[r].double().abs() @ w1[e].double().abs().T), (hidden + 8) * U * (rows[r].double().abs() @ w3[e].double().abs().T)
        s = torch.nn.functional.silu(gd)
        off = H * (SILU_SLOPE * gd.abs() * ud.abs() + s.abs() * ud.abs()) + 2 * H * (s * ud).abs()
        off += 2 * (SILU_SLOPE * sums[0] * ud.abs() + s.abs() * sums[1])
        m = w2[e].double().abs().T
        off = off @ m + 2 * (ffn + 8) * U * ((s * ud).abs() @ m) + H * ((s * ud) @ w2[e].double().T).abs()
        bound.index_add_(0, order[r] // k, off * weight[r].double()[:, None])
        value.index_add_(0, order[r] // k, ((s * ud) @ w2[e].double().T) * weight[r].double()[:, None])
    assert ((y - fused.double()).abs() <= 1.04 * bound + H * value.abs() + 1e-30).all()
    assert ((y - value).abs() <= 1.04 * bound + 1e-30).all()


@pytest.mark.parametrize("counts,D,F", [([40, 0, 100], 128, 192), ([2, 1, 3], 256, 128), ([300, 700, 11], 192, 256)])
def test_a_training_step_of_experts(counts, D, F):
    """Two micro-batches through w2 silu(w1 x) u, u = w3 x, and back, in fp32, gradients of the weights accumulated, against 64 bits.  With G = |x| |w1|,
    V = |x| |w3| and Q = |dy| |w2|: g and u are off by (D + 8) u of G and V, dh by (D + 8) u of Q, so dg = dh u silu'(g) by u of
    Q V ((D + 8) (1.1 + 1.1 + G / 2) + 16), du = dh silu(g) by u of Q G ((D + 8) 2.1 + 16), the activations by u of G V (2.1 (D + 8) + 16); the sums
    of the gradients add their lengths."""
    E = len(counts)
    o, offsets = table(counts)
    R = o[-1]
    w1, w3, w2 = (normal(E, *s, seed=3 + i, std=0.08) for i, s in enumerate(((F, D), (F, D), (D, F))))
    ws = workspace(E, F, D, F32, R)
    grads = [torch.empty_like(w) for w in (w1, w3, w2)]
    exact = [torch.zeros(w.shape, dtype=torch.float64, device=DEV) for w in (w1, w3, w2)]
    sizes = [torch.zeros_like(e) for e in exact]
    for batch in range(2):
        x, dy = normal(R, D, seed=10 + batch), normal(R, D, seed=20 + batch)
        g, v, dh = (torch.empty(R, F, device=DEV) for _ in range(3))
        y, dx, part = (torch.empty(R, D, device=DEV) for _ in range(3))
        products.moe_grouped_product(x, offsets, w1, g, ws)
        products.moe_grouped_product(x, offsets, w3, v, ws)
        s = torch.sigmoid(g)
        act = g * s * v
        products.moe_grouped_product(act, offsets, w2, y, ws)
        products.moe_grouped_product_dgrad(dy, offsets, w2, dh, ws)
        dg, dv = dh * v * (s + g * s * (1 - s)), dh * g * s
        products.moe_grouped_product_wgrad(dg, x, offsets, grads[0], batch > 0, ws)
        products.moe_grouped_product_wgrad(dv, x, offsets, grads[1], batch > 0, ws)
        products.moe_grouped_product_wgrad(dy, act, offsets, grads[2], batch > 0, ws)
        products.moe_grouped_product_dgrad(dg, offsets, w1, dx, ws)
        products.moe_grouped_product_dgrad(dv, offsets, w3, part, ws)
        dx += part
        for e in range(E):
            r, n = slice(o[e], o[e + 1]), counts[e]
            leaves = [t.detach().double().requires_grad_() for t in (x[r], w1[e], w3[e], w2[e])]
            gd = leaves[0] @ leaves[1].T
            out = (torch.nn.functional.silu(gd) * (leaves[0] @ leaves[2].T)) @ leaves[3].T
            out.backward(dy[r].double())
            xa, w1a, w3a, w2a, dya = (t.double().abs() for t in (x[r], w1[e], w3[e], w2[e], dy[r]))
            G, V, Q = xa @ w1a.T, xa @ w3a.T, dya @ w2a
            off_g = Q * V * ((D + 8) * (2 * SILU_SLOPE + SILU_BEND * G) + 16)
            off_v = Q * G * ((D + 8) * (1 + SILU_SLOPE) + 16)
            off_a = G * V * ((D + 8) * (1 + SILU_SLOPE) + 16)
            assert ((y[r].double() - out).abs() <= 1.01 * U * ((off_a + (F + 8) * G * V) @ w2a.T)).all(), f"y of expert {e}"
            dx_bound = (off_g + (F + 10) * SILU_SLOPE * Q * V) @ w1a + (off_v + (F + 10) * Q * G) @ w3a
            assert ((dx[r].double() - leaves[0].grad).abs() <= 1.01 * U * dx_bound).all(), f"dx of expert {e}"
            for i, (bound, big) in enumerate(((off_g, SILU_SLOPE * Q * V), (off_v, Q * G))):
                sizes[i][e] += (bound + (2 * n + 10) * big).T @ xa
            sizes[2][e] += dya.T @ (off_a + (2 * n + 10) * G * V)
            for total, leaf in zip(exact, leaves[1:]):
                total[e] += leaf.grad
    for name, got, want, size in zip(("w1", "w3", "w2"), grads, exact, sizes):
        assert ((got.double() - want).abs() <= 1.01 * U * size).all(), name


@pytest.mark.parametrize("T,E,k,hidden,ffn", [(2, 8, 2, 320, 256), (120, 8, 2, 256, 448), (700, 4, 2, 640, 320)])
def test_experts_in_8_bits(T, E, k, hidden, ffn):
    """Quantised rows and weights through both products of an expert; every step against its formula on what the step before left."""
    x, _, _, order, offsets = selections(T, E, k, hidden, seed=30)
    o, R = offsets.tolist(), T * k
    rows = x[order // k].contiguous()
    ws = workspace(E, ffn, hidden, BF16, R)

    def quantised_weights(w):
        E, N, K = w.shape
        q, s = torch.empty(E, N, K, dtype=torch.uint8, device=DEV), torch.empty(E, -(-N // 128), -(-K // 128), device=DEV)
        products.moe_quantize_weights_fp8(w, q, s)
        return q, s

    def product(x, w):
        (R, K), (E, N, _) = x.shape, w.shape
        kb = -(-K // 128)
        xq, xs = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, kb, device=DEV)
        products.moe_quantize_rows_fp8(x, xq, xs)
        want, scale = quantised(x, 1)
        assert same_bits(xq, want) and torch.equal(xs.double(), scale)
        wq, wsc = quantised_weights(w)
        y = torch.full((R, N), UNTOUCHED, dtype=BF16, device=DEV)
        products.moe_grouped_product_fp8(xq, xs, offsets, wq, wsc, y, ws)
        values = want * scale.repeat_interleave(128, 1)[:, :K]
        for e in range(E):
            r = slice(o[e], o[e + 1])
            m = wq[e].view(torch.float8_e4m3fn).double() * wsc[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
            exact, size = values[r] @ m.T, values[r].abs() @ m.abs().T
            assert ((y[r].double() - exact).abs() <= (2.0 ** -12 + (kb + 8) * U) * size + H * exact.abs()).all(), f"expert {e}"
        return y

    up = product(rows, normal(E, 2 * ffn, hidden, dtype=BF16, seed=41, std=0.06))
    act = (torch.nn.functional.silu(up[:, :ffn].float()) * up[:, ffn:].float()).to(BF16)
    product(act, normal(E, hidden, ffn, dtype=BF16, seed=42, std=0.06))


# ---- every way in which a call is cut

FORWARD = [   # rows of each expert, N, K: tiles of every height, several rounds, cut tiles, many passes of the few-row kernel
    ([1, 1], 192, 8256),                       # eight wavefronts share the contraction
    ([3] * 5, 128, 8192),
    ([15, 0, 30, 16, 9], 256, 320),            # two row fragments a pass
    ([0, 0, 0, 77, 0, 0, 0, 1], 192, 256),     # more rows than a pass
    ([20, 64, 70, 100, 130, 170, 200, 250], 576, 192),
    ([33, 65, 97, 129, 161, 193, 225, 256, 257, 300], 256, 64),
    ([1500, 900, 260, 90, 7, 0, 3, 40], 4160, 128),     # several rounds, the last one cut or not
    ([2300, 1800], 2112, 448),
    ([150, 60], 512, 8256),                    # few tiles, a long contraction: cut
    ([500] * 9, 1024, 1024),
    ([40 + 7 * i for i in range(64)], 320, 192),
    # sizes of the large tiles: every height, a ragged last feature tile, one round and several, cut and whole
    ([20, 64, 70, 100, 130, 170, 200, 250], 2112, 4160),
    ([33, 65, 97, 129, 161, 193, 225, 256, 257, 300], 4160, 2112),
    ([1500, 900, 260, 90, 7, 0, 3, 40], 4160, 1088),
    ([600], 2624, 8256),
    ([5000, 0, 77], 3200, 1216),
    # and their neighbours in tiles of 64
    ([1, 64, 65, 0, 128, 200], 320, 4608),
    ([63], 64, 64),
    ([130, 2, 0, 61], 1088, 1088),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,N,K", FORWARD)
def test_rows_are_cut_in_every_way(counts, N, K, dtype):
    """Forward, and the gradient of a product with exchanged features, which is cut alike."""
    o, offsets = table(counts, 2)
    R, E = o[-1] + 3, len(counts)
    x, w, w_t = normal(R, K, dtype=dtype, seed=1), normal(E, N, K, dtype=dtype, seed=3), normal(E, K, N, dtype=dtype, seed=4)
    ws = workspace(E, N, K, dtype, R)
    y, dx = (torch.full((R, N), UNTOUCHED, dtype=dtype, device=DEV) for _ in range(2))
    products.moe_grouped_product(x, offsets, w, y, ws)
    products.moe_grouped_product_dgrad(x, offsets, w_t, dx, ws)
    for form, got, m in (("forward", y, w), ("dgrad", dx, w_t)):
        assert (got[:2] == UNTOUCHED).all() and (got[-3:] == UNTOUCHED).all()
        for r, want, size in reference(form, o, x, m):
            check(got[r], want, size, K, dtype, f"{form} rows {r.start}-{r.stop}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,N,K", [
    ([3000, 1, 0, 500], 320, 192),             # few tiles and many rows: cut
    ([64, 128, 192, 256, 193, 65], 64, 320),
    ([700, 0, 701, 20], 448, 576),
    ([300] * 12, 1088, 1088),                  # several rounds
    ([9000], 128, 64),
    ([5 * i for i in range(64)], 192, 128),
    # sizes of the large tiles: whole, cut, ragged, without rows
    ([700, 0, 701, 20], 2112, 2112),
    ([3000], 3136, 3136),
    ([500, 3, 0, 64, 1], 3136, 1600),
    ([63, 65, 0, 1, 128, 127, 129, 40] * 8, 512, 320),
])
def test_matrices_gradients_are_cut_in_every_way(counts, N, K, dtype):
    o, offsets = table(counts, 1)
    R, E = o[-1] + 2, len(counts)
    x, dy = normal(R, K, dtype=dtype, seed=1), normal(R, N, dtype=dtype, seed=2)
    ws = workspace(E, N, K, dtype, R)
    want = reference("wgrad", o, dy, x)
    for out_dtype, accumulate in {(dtype, False), (F32, False), (F32, True)}:
        dw = normal(E, N, K, seed=4) if accumulate else torch.full((E, N, K), UNTOUCHED, dtype=out_dtype, device=DEV)
        old = dw.double() if accumulate else torch.zeros(E, N, K, dtype=torch.float64, device=DEV)
        products.moe_grouped_product_wgrad(dy, x, offsets, dw, accumulate, ws)
        for e, value, size in want:
            check(dw[e], old[e] + value, old[e].abs() + size, counts[e] + 1, out_dtype, f"{out_dtype} {accumulate} expert {e}")


@pytest.mark.parametrize("counts,N,K", FORWARD + [
    ([400, 200], 256, 8256),                   # an odd number of blocks, the last one of 64, cut
    ([1000, 30], 704, 1152),                   # nine blocks
    ([5, 0, 300], 128, 128),                   # one block
    ([20] * 16, 1024, 1024),                   # four feature fragments in the few-row kernel
    ([33 * i for i in range(1, 9)], 320, 704),
])
def test_fp8_rows_are_cut_in_every_way(counts, N, K):
    """Integers of four bits: the sums inside a block lose nothing.  The scales behind every row's last one are NaN in the row of nobody."""
    o, offsets = table(counts, 1)
    R, E, kb, nb = o[-1] + 1, len(counts), -(-K // 128), -(-N // 128)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    xq, wq = (torch.randint(-15, 16, s, device=DEV, generator=g).float().to(torch.float8_e4m3fn) for s in ((R, K), (E, N, K)))
    xs, wsc = (torch.exp(torch.randn(s, device=DEV, generator=g)) for s in ((R, kb), (E, nb, kb)))
    xs[-1] = xs[0] = math.nan
    y = torch.full((R, N), UNTOUCHED, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, wsc, y, workspace(E, N, K, BF16, R))
    assert (y[0] == UNTOUCHED).all() and (y[-1] == UNTOUCHED).all()
    x = xq.double() * xs.double().repeat_interleave(128, 1)[:, :K]
    for e in range(E):
        r = slice(o[e], o[e + 1])
        m = wq[e].double() * wsc[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        check(y[r], x[r] @ m.T, x[r].abs() @ m.abs().T, kb, BF16, f"expert {e}")


@pytest.mark.parametrize("R,N,K", [(40, 320, 384), (300, 256, 640), (5, 64, 128), (1500, 4160, 1152), (300, 4160, 4480)])
def test_a_row_of_bad_scales_reaches_no_other(R, N, K):
    """Blocks in odd numbers: behind a row's last scale lies the next row's first, which is NaN or infinite here in every other row."""
    x, w = normal(R, K, dtype=BF16, seed=1), normal(1, N, K, dtype=BF16, seed=3)
    x[1::2, 0] = math.nan
    xq, xs = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, K // 128, device=DEV)
    wq, wsc = torch.empty(1, N, K, dtype=torch.uint8, device=DEV), torch.empty(1, -(-N // 128), K // 128, device=DEV)
    products.moe_quantize_rows_fp8(x, xq, xs)
    products.moe_quantize_weights_fp8(w, wq, wsc)
    for bad in (math.nan, math.inf):
        xs[1::2, 0] = bad
        y = torch.zeros(R, N, dtype=BF16, device=DEV)
        products.moe_grouped_product_fp8(xq, xs, None, wq, wsc, y, workspace(1, N, K, BF16, R))
        assert torch.isfinite(y[0::2]).all() and torch.isnan(y[1::2]).all()


# ---- calls beside and behind one another

class Calls:
    """One of each call on fixed buffers."""

    def __init__(self, counts, N, K, dtype, seed, ws=None):
        self.E, self.N, self.K, self.dtype = len(counts), N, K, dtype
        o, self.offsets = table(counts)
        self.R = o[-1]
        self.x, self.dy = normal(self.R, K, dtype=dtype, seed=seed), normal(self.R, N, dtype=dtype, seed=seed + 1)
        self.w = normal(self.E, N, K, dtype=dtype, seed=seed + 2)
        self.ws = workspace(self.E, N, K, dtype, self.R) if ws is None else ws
        kb, nb = -(-K // 128), -(-N // 128)
        self.q, self.s = torch.empty(self.R, K, dtype=torch.uint8, device=DEV), torch.empty(self.R, kb, device=DEV)
        self.wq, self.wq_s = torch.empty(self.E, N, K, dtype=torch.uint8, device=DEV), torch.empty(self.E, nb, kb, device=DEV)
        self.y, self.dx = torch.empty(self.R, N, dtype=dtype, device=DEV), torch.empty(self.R, K, dtype=dtype, device=DEV)
        self.dw, self.y8 = torch.empty(self.E, N, K, device=DEV), torch.empty(self.R, N, dtype=BF16, device=DEV)

    def __call__(self):
        products.moe_grouped_product(self.x, self.offsets, self.w, self.y, self.ws)
        products.moe_grouped_product_dgrad(self.dy, self.offsets, self.w, self.dx, self.ws)
        products.moe_grouped_product_wgrad(self.dy, self.x, self.offsets, self.dw, False, self.ws)
        products.moe_grouped_product_wgrad(self.dy, self.x, self.offsets, self.dw, True, self.ws)
        products.moe_quantize_rows_fp8(self.x, self.q, self.s)
        products.moe_quantize_weights_fp8(self.w, self.wq, self.wq_s)
        if self.dtype == BF16:
            products.moe_grouped_product_fp8(self.q, self.s, self.offsets, self.wq, self.wq_s, self.y8, self.ws)

    def outputs(self):
        return [self.y, self.dx, self.dw, self.q, self.s.view(torch.int32), self.wq, self.wq_s.view(torch.int32)] + ([self.y8] if self.dtype == BF16 else [])

    def spoil(self):
        for t in self.outputs():
            t.fill_(3)
        self.ws.fill_(0xFF)

    def results(self):
        return [t.clone() for t in self.outputs()]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b, strict=True))


MIXED = [([300, 0, 40, 9], 512, 704), ([2, 1, 0, 1], 256, 1024), ([700, 0, 300, 65], 2112, 4160)]   # small tiles, few rows, large tiles


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,N,K", MIXED)
def test_results_are_the_same_every_time(counts, N, K, dtype):
    c = Calls(counts, N, K, dtype, 50)
    c()
    first = c.results()
    for byte in (0x00, 0xFF, 0x7F):
        c.spoil()
        c.ws.fill_(byte)
        c()
        assert same(c.outputs(), first)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,N,K", MIXED)
def test_graphs_are_replayed(counts, N, K, dtype):
    """Two graphs of all calls with one workspace, replayed in turn with other inputs and tables, eager calls with that workspace between them."""
    a = Calls(counts, N, K, dtype, 60)
    b = Calls(list(reversed(counts)), N, K, dtype, 70, a.ws)
    a()   # (everything is loaded before the capture)
    torch.cuda.synchronize()
    graphs = []
    for c in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c()
        graphs.append(graph)
    for n in range(3):
        for c, graph in zip((a, b), graphs):
            c.x.copy_(normal(c.R, K, dtype=dtype, seed=80 + n))
            c.offsets.copy_(table(counts if n % 2 else list(reversed(counts)))[1])
            c()
            want = c.results()
            c.spoil()
            graph.replay()
            torch.cuda.synchronize()
            assert same(c.outputs(), want), f"replay {n}"


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_streams_of_their_own(dtype):
    """Two streams at once, each with its workspace, and inputs that the stream itself has just written."""
    calls = [Calls(*shape, dtype, 90 + 10 * i) for i, shape in enumerate(MIXED)]
    want = []
    for c in calls:
        c()
        want.append(c.results())
    inputs = [c.x.clone() for c in calls]
    for c in calls:
        c.spoil()
        c.x.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for c, x, s in zip(calls, inputs, streams):
            with torch.cuda.stream(s):
                c.x.copy_(x)
                c()
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert same(c.outputs(), w)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,N,K", [([30, 0, 100, 3], 320, 448), ([300, 0, 700, 3], 2112, 4160)])
def test_buffers_begin_at_any_16_bytes(counts, N, K, dtype):
    """Operands and results inside larger buffers, 16 bytes into them, with NaN around."""
    o, offsets = table(counts)
    R, E, skip = o[-1], len(counts), 16 // torch.tensor([], dtype=dtype).element_size()

    def inside(*shape, dt=dtype, seed=None):
        n, at = math.prod(shape), 16 // torch.tensor([], dtype=dt).element_size()
        buffer = torch.full((n + 2 * at,), math.nan, dtype=dt, device=DEV)
        if seed is not None:
            buffer[at:at + n] = normal(*shape, dtype=dt, seed=seed).flatten()
        return buffer, buffer[at:at + n].view(shape)

    x, dy, w = inside(R, K, seed=1)[1], inside(R, N, seed=2)[1], inside(E, N, K, seed=3)[1]
    outs = [inside(R, N), inside(R, K), inside(E, N, K, dt=F32)]
    ws = workspace(E, N, K, dtype, R)
    products.moe_grouped_product(x, offsets, w, outs[0][1], ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, outs[1][1], ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, outs[2][1], False, ws)
    for buffer, t in outs:
        assert torch.isfinite(t).all() and int(torch.isnan(buffer).sum()) == buffer.numel() - t.numel()
    for (form, a, b, depth), (_, got) in zip((("forward", x, w, K), ("dgrad", dy, w, N)), outs):
        for r, want, size in reference(form, o, a, b):
            check(got[r], want, size, depth, dtype, form)
    for e, value, size in reference("wgrad", o, dy, x):
        check(outs[2][1][e], value, size, counts[e], F32, "wgrad")
    assert skip * x.element_size() == 16


# ---- buffers that 32 bits do not reach

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("few", [True, False])
def test_rows_and_matrices_behind_2_to_the_32(dtype, few):
    """The last rows of x and dx and the last of 64 matrices lie more than 2^32 elements into their buffers."""
    E, N, K = 64, 4096, 16448
    assert E * N * K > 1 << 32
    n = 3 if few else 200
    R = 40 if few else (1 << 32) // K + 300   # (few: only the matrices are large)
    before = R - n - 2
    offsets = torch.tensor([before, before + 2] + [before + 2] * (E - 2) + [R], dtype=torch.int32, device=DEV)
    w = torch.empty(E, N, K, dtype=dtype, device=DEV)
    w[0], w[-1] = normal(N, K, dtype=dtype, seed=1), normal(N, K, dtype=dtype, seed=2)
    x, dx = torch.empty(R, K, dtype=dtype, device=DEV), torch.full((R, K), UNTOUCHED, dtype=dtype, device=DEV)
    dy, y = normal(R, N, dtype=dtype, seed=4), torch.empty(R, N, dtype=dtype, device=DEV)
    x[before:] = normal(n + 2, K, dtype=dtype, seed=3)
    ws = workspace(E, N, K, dtype, R)
    products.moe_grouped_product(x, offsets, w, y, ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx, ws)
    parts = [(slice(before, before + 2), 0), (slice(before + 2, R), E - 1)]
    for r, e in parts:
        m = w[e].double()
        check(y[r], x[r].double() @ m.T, x[r].double().abs() @ m.abs().T, K, dtype, f"expert {e}")
        check(dx[r], dy[r].double() @ m, dy[r].double().abs() @ m.abs(), N, dtype, f"dx, expert {e}")
    assert (dx[before - 1] == UNTOUCHED).all()
    del y, dx, m
    dw = w if dtype == F32 else torch.empty(E, N, K, device=DEV)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)
    for r, e in parts:
        a, b = dy[r].double(), x[r].double()
        check(dw[e], a.T @ b, a.abs().T @ b.abs(), r.stop - r.start, F32, f"dw, expert {e}")
    assert not dw[1].any() and not dw[E - 2].any()


@pytest.mark.parametrize("few", [True, False])
def test_8_bit_numbers_behind_2_to_the_32(few):
    E, N, K = 64, 4096, 16448
    n = 3 if few else 300
    R = 40 if few else (1 << 32) // K + 400   # (few: only the matrices are large)
    before = R - n - 2
    offsets = torch.tensor([before, before + 2] + [before + 2] * (E - 2) + [R], dtype=torch.int32, device=DEV)
    x, w = torch.zeros(R, K, dtype=BF16, device=DEV), torch.zeros(E, N, K, dtype=BF16, device=DEV)
    x[before:] = normal(n + 2, K, dtype=BF16, seed=3)
    w[0], w[-1] = normal(N, K, dtype=BF16, seed=1), normal(N, K, dtype=BF16, seed=2)
    kb, nb = -(-K // 128), N // 128
    xq, xs = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, kb, device=DEV)
    wq, wsc = torch.empty(E, N, K, dtype=torch.uint8, device=DEV), torch.empty(E, nb, kb, device=DEV)
    wq_t, wsc_t = torch.empty(E, K, N, dtype=torch.uint8, device=DEV), torch.empty(E, kb, nb, device=DEV)
    products.moe_quantize_rows_fp8(x, xq, xs)
    products.moe_quantize_weights_fp8(w, wq, wsc, wq_t, wsc_t)
    numbers, scale = quantised(x[-2:], 1)
    assert same_bits(xq[-2:], numbers) and torch.equal(xs[-2:].double(), scale)
    numbers, scale = quantised(w[-1], 128)
    assert same_bits(wq[-1], numbers) and torch.equal(wsc[-1].double(), scale)
    assert torch.equal(wq_t[-1], wq[-1].T) and torch.equal(wsc_t[-1], wsc[-1].T)
    y = torch.empty(R, N, dtype=BF16, device=DEV)
    products.moe_grouped_product_fp8(xq, xs, offsets, wq, wsc, y, workspace(E, N, K, BF16, R))
    values = xq[before:].view(torch.float8_e4m3fn).double() * xs[before:].double().repeat_interleave(128, 1)[:, :K]
    for r, e in ((slice(0, 2), 0), (slice(2, n + 2), E - 1)):
        m = wq[e].view(torch.float8_e4m3fn).double() * wsc[e].double().repeat_interleave(128, 0).repeat_interleave(128, 1)[:, :K]
        want, size = values[r] @ m.T, values[r].abs() @ m.abs().T
        off = (y[before:][r].double() - want).abs()
        assert (off <= (2.0 ** -12 + (kb + 8) * U) * size + H * want.abs()).all(), f"expert {e}"


def test_layouts_are_refused():
    x, w, y = normal(8, 128, dtype=BF16), normal(2, 64, 128, dtype=BF16), torch.empty(8, 64, dtype=BF16, device=DEV)
    o, ws = torch.tensor([0, 4, 8], dtype=torch.int32, device=DEV), workspace(2, 64, 128, BF16, 8)
    products.moe_grouped_product(x, o, w, y, ws)
    for bad in (dict(x=normal(128, 8, dtype=BF16).T), dict(x=normal(16, 128, dtype=BF16)[::2]), dict(w=normal(2, 128, 64, dtype=BF16).transpose(1, 2)),
                dict(o=o[:2]), dict(y=y[:4]), dict(w=w.cpu()), dict(ws=ws.cpu())):
        a = dict(x=x, o=o, w=w, y=y, ws=ws) | bad
        with pytest.raises(ValueError):
            products.moe_grouped_product(*a.values())
    for bad in (dict(o=o.long()), dict(w=w.float()), dict(y=y.float()), dict(x=x.half())):
        a = dict(x=x, o=o, w=w, y=y, ws=ws) | bad
        with pytest.raises(TypeError):
            products.moe_grouped_product(*a.values())
    with pytest.raises(moe.MoeError):   # two experts need a table
        products.moe_grouped_product(x, None, w, y, ws)
    with pytest.raises(moe.MoeError):
        products.moe_grouped_product(x, o, w, y, ws[:1024])
    with pytest.raises(moe.MoeError):   # not at 16 bytes
        products.moe_grouped_product(normal(9 * 128, dtype=BF16)[4:4 + 8 * 128].view(8, 128), o, w, y, ws)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,N,K", [(9, 192, 448), (700, 192, 448), (700, 2112, 4160)])
@pytest.mark.parametrize("values", [[-7, 3, 5, 9], [0, 1 << 30, 2, 1 << 30], [0, 6, 0, 6], [1 << 30] * 4, [-(1 << 31), -1, 4, 4], [5, 5, 5, 5]])
def test_tables_of_any_values_stay_inside_the_buffers(values, R, N, K, dtype):
    """Every call on tables that leave the rows or do not ascend: nothing behind the buffers is written, and what ascends is computed."""
    E, guard, kb, nb = 3, 64, -(-K // 128), -(-N // 128)
    offsets = torch.tensor(values, dtype=torch.int32, device=DEV)
    x, dy, w = normal(R, K, dtype=dtype, seed=1), normal(R, N, dtype=dtype, seed=2), normal(E, N, K, dtype=dtype, seed=3)
    ws = workspace(E, N, K, dtype, R)
    y, dx = (torch.full((R + guard, n), UNTOUCHED, dtype=dtype, device=DEV) for n in (N, K))
    dw = torch.full((E + 1, N, K), UNTOUCHED, device=DEV)
    products.moe_grouped_product(x, offsets, w, y[:R], ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx[:R], ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw[:E], False, ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw[:E], True, ws)
    if dtype == BF16:
        q, s = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, kb, device=DEV)
        wq, wsc = torch.empty(E, N, K, dtype=torch.uint8, device=DEV), torch.empty(E, nb, kb, device=DEV)
        y8 = torch.full((R + guard, N), UNTOUCHED, dtype=BF16, device=DEV)
        products.moe_quantize_rows_fp8(x, q, s)
        products.moe_quantize_weights_fp8(w, wq, wsc)
        products.moe_grouped_product_fp8(q, s, offsets, wq, wsc, y8[:R], ws)
        assert (y8[R:] == UNTOUCHED).all()
    assert (y[R:] == UNTOUCHED).all() and (dx[R:] == UNTOUCHED).all() and (dw[E] == UNTOUCHED).all()
    o = [min(max(v, 0), R) for v in values]
    if o == sorted(o):
        for form, got, a, depth in (("forward", y, x, K), ("dgrad", dx, dy, N)):
            for r, want, size in reference(form, o, a, w):
                check(got[r], want, size, depth, dtype, form)
        for e, value, size in reference("wgrad", o, dy, x):
            check(dw[e], 2 * value, 2 * size, 2 * (o[e + 1] - o[e]) + 1, F32, "wgrad, added to itself")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,K", [(1 << 20, 64), (64, 1 << 20)])
@pytest.mark.parametrize("counts", [[3, 2], [40, 300]])
def test_the_longest_rows(counts, N, K, dtype):
    """Features at their limit, either way, through every call."""
    o, offsets = table(counts)
    R, E = o[-1], 2
    x, dy, w = normal(R, K, dtype=dtype, seed=1), normal(R, N, dtype=dtype, seed=2), normal(E, N, K, dtype=dtype, seed=3)
    ws = workspace(E, N, K, dtype, R)
    y, dx, dw = torch.empty(R, N, dtype=dtype, device=DEV), torch.empty(R, K, dtype=dtype, device=DEV), torch.empty(E, N, K, device=DEV)
    products.moe_grouped_product(x, offsets, w, y, ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx, ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)
    for form, got, a, depth in (("forward", y, x, K), ("dgrad", dx, dy, N)):
        for r, want, size in reference(form, o, a, w):
            check(got[r], want, size, depth, dtype, form)
    for e, value, size in reference("wgrad", o, dy, x):
        check(dw[e], value, size, counts[e], F32, "wgrad")
    if dtype == F32:
        return
    kb, nb = -(-K // 128), -(-N // 128)
    q, s = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, kb, device=DEV)
    wq, wsc = torch.empty(E, N, K, dtype=torch.uint8, device=DEV), torch.empty(E, nb, kb, device=DEV)
    products.moe_quantize_rows_fp8(x, q, s)
    products.moe_quantize_weights_fp8(w, wq, wsc)
    products.moe_grouped_product_fp8(q, s, offsets, wq, wsc, y, ws)
    values = q.view(torch.float8_e4m3fn).double() * s.double().repeat_interleave(128, 1)[:, :K]
    for e in range(E):
        r = slice(o[e], o[e + 1])
        m = wq[e].view(torch.float8_e4m3fn).double() * wsc[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        want, size = values[r] @ m.T, values[r].abs() @ m.abs().T
        assert ((y[r].double() - want).abs() <= (2.0 ** -12 + (kb + 8) * U) * size + H * want.abs()).all(), f"8 bits, expert {e}"


@pytest.mark.parametrize("counts,N,K", [([70, 31, 145], 320, 448), ([600, 31, 450], 2112, 4160)])
def test_not_a_number_stays_with_its_rows_and_expert_in_every_tile(counts, N, K):
    """NaN in a row, in an expert's matrix and behind the last row, small tiles and large: what the formulas say and nothing else."""
    o, offsets = table(counts)
    R = o[-1] + 3
    x, dy, w = normal(R, K, dtype=BF16, seed=1), normal(R, N, dtype=BF16, seed=2), normal(3, N, K, dtype=BF16, seed=3)
    x[o[-1]:], dy[o[-1]:] = math.nan, math.inf
    x[o[1] + 5, 7], w[2, 70, 100] = math.nan, math.inf
    ws = workspace(3, N, K, BF16, R)
    y, dx, dw = torch.zeros(R, N, dtype=BF16, device=DEV), torch.zeros(R, K, dtype=BF16, device=DEV), torch.zeros(3, N, K, device=DEV)
    products.moe_grouped_product(x, offsets, w, y, ws)
    products.moe_grouped_product_dgrad(dy, offsets, w, dx, ws)
    products.moe_grouped_product_wgrad(dy, x, offsets, dw, False, ws)
    bad_y, bad_dx, bad_dw = (torch.zeros(t.shape, dtype=torch.bool, device=DEV) for t in (y, dx, dw))
    bad_y[o[1] + 5], bad_y[o[2]:o[3], 70] = True, True
    bad_dx[o[2]:o[3], 100] = True
    bad_dw[1, :, 7] = True
    for got, bad in ((y, bad_y), (dx, bad_dx), (dw, bad_dw)):
        assert torch.equal(~torch.isfinite(got), bad)
    kb, nb = -(-K // 128), -(-N // 128)
    q, s = torch.empty(R, K, dtype=torch.uint8, device=DEV), torch.empty(R, kb, device=DEV)
    wq, wsc = torch.empty(3, N, K, dtype=torch.uint8, device=DEV), torch.empty(3, nb, kb, device=DEV)
    products.moe_quantize_rows_fp8(x, q, s)
    products.moe_quantize_weights_fp8(w, wq, wsc)
    y.zero_()
    products.moe_grouped_product_fp8(q, s, offsets, wq, wsc, y, ws)
    bad_y[o[2]:o[3], :128] = True    # (a tile of an expert's matrix)
    assert torch.equal(~torch.isfinite(y), bad_y)
