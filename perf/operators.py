"""Performance cases of the products grouped by expert and of their 8-bit form.

A case is one pass through one of the operators on inputs that are resident in GPU memory:
  product    y[r] = W_e x[r] for every row r of expert e (rows sorted by expert, ragged)
  gradients  the gradients of that product: dx[r] = W_e^T dy[r] and dW_e = sum_r dy[r] x[r]^T
  rows       rows of activations to e4m3 with a scale for each 128 values of a row
  weights    weights to e4m3 with a scale for each 128 x 128 tile, and the same values transposed
  fp8        the product of such rows and weights, grouped by expert or (one expert) dense
The shapes are those of the benchmark: experts of the Mixtral-8x7B-shaped layer (hidden 4096, 8 experts of
width 14336, top-2, Zipf 1.2 routing skew), of the Phi-3.5-MoE-shaped one (16 of width 6400, Zipf 1.5), of the
fine-grained one (hidden 2048, 64 of width 1408, top-6, Zipf 0.5) and of the tiny fp32 configuration.

With `own` the framework's entry points are called; without, the same is computed with elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BLOCK = 128
_E4M3_MAX = 448.0
_LEAST_AMAX = 2.0 ** -60   # a block of smaller values is scaled as if this were its largest


def _case(name, kind, experts, n, k, rows, dtype="bf16", zipf=0.0, **more):
    return dict(more, name=name, kind=kind, experts=experts, n=n, k=k, rows=rows, dtype=dtype, zipf=zipf)


def listed():
    return [
        # the exact-arithmetic configuration at its own size: 64 tokens, top-2; latency counts
        _case("product_f32_tiny", "product", 8, 512, 256, 128, "f32", 1.2),
        # one decoded token through the up-projection of its two experts: a stream over their weights
        _case("product_decode_mixtral", "product", 8, 14336, 4096, 2, "bf16", 1.2),
        # the down-projection of a prompt of 4096 tokens
        _case("product_prefill_mixtral", "product", 8, 4096, 14336, 8192, "bf16", 1.2),
        # gradients in fp32 at odd row counts, as a check of a bf16 run makes them
        _case("gradients_f32_odd", "gradients", 16, 1408, 2048, 1030, "f32", 0.8, dw="f32"),
        # many small experts: 1003 tokens, top-6, ragged groups of under a hundred rows; gradients kept in the weights' type
        _case("gradients_finegrained", "gradients", 64, 1408, 2048, 6018, "bf16", 0.5, dw="bf16"),
        # a training step's largest products: 4096 tokens, top-2, the weights' gradient in fp32
        _case("gradients_mixtral", "gradients", 8, 14336, 4096, 8192, "bf16", 1.2, dw="f32"),
        # activations of a decode batch of 32 tokens before the down-projection, and of a prompt
        _case("rows_decode", "rows", 1, 0, 14336, 64),
        _case("rows_prefill", "rows", 1, 0, 14336, 8192),
        # a layer's weights when they are loaded, or after an optimizer step
        _case("weights_phi", "weights", 16, 6400, 4096, 0),
        # one decoded token in 8 bits
        _case("fp8_decode_phi", "fp8", 16, 6400, 4096, 2, "bf16", 1.5),
        # a batch of 77 decoding sequences, every expert with a few rows
        _case("fp8_batch_mixtral", "fp8", 8, 14336, 4096, 154, "bf16", 1.2),
        # a prompt of 4096 tokens in 8 bits
        _case("fp8_prefill_mixtral", "fp8", 8, 14336, 4096, 8192, "bf16", 1.2),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(("product", "product", "gradients", "gradients", "rows", "weights", "fp8", "fp8", "fp8"))
    experts = rng.choice((1, 2, 4, 8, 12, 16, 33, 64))
    n, k = 64 * _log_uniform(rng, 1, 224), 64 * _log_uniform(rng, 1, 224)
    if rng.random() < 0.5:   # widths of the workloads above
        n, k = rng.choice(((14336, 4096), (4096, 14336), (6400, 4096), (4096, 6400), (1408, 2048), (2048, 1408), (512, 256)))
    rows = _log_uniform(rng, 1, 8192)
    if kind == "rows":
        experts, n = 1, 0
    dtype = "f32" if rng.random() < 0.25 and kind != "fp8" else "bf16"   # (the 8-bit product's result is bf16)
    most = 8 * 14336 * 4096   # weights of the largest listed case
    while experts * n * k > most:
        experts = max(1, experts // 2)
    if dtype == "f32" and kind in ("product", "gradients"):
        rows = min(rows, 1030)
        while experts * n * k > most // 2:
            experts = max(1, experts // 2)
    if rows * n * k > 8192 * 14336 * 4096:
        rows = 8192 * 14336 * 4096 // (n * k)
    more = {"dw": rng.choice(("f32", dtype))} if kind == "gradients" else {}
    return dict(more, kind=kind, experts=experts, n=n, k=k, rows=0 if kind == "weights" else rows, dtype=dtype,
                zipf=rng.choice((0.0, 0.5, 1.2)))


def _offsets(case, seed):
    """Rows of each expert: the routing of a skewed gate, experts in no order of popularity, some without rows where there are few."""
    rng = np.random.RandomState(seed % (1 << 31))
    p = np.arange(1, case["experts"] + 1, dtype=np.float64) ** -case["zipf"]
    p = rng.permutation(p / p.sum())
    return [0] + np.cumsum(rng.multinomial(case["rows"], p)).tolist()


def prepare(case, seed):
    """Inputs on the GPU, output buffers and, as the plan of the plain form, which rows are whose."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    E, N, K, R, dtype, kind = case["experts"], case["n"], case["k"], case["rows"], _DTYPES[case["dtype"]], case["kind"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, device="cuda", generator=gen).mul_(std).to(dtype)

    def empty(*shape, dtype=dtype):
        return torch.empty(shape, device="cuda", dtype=dtype)

    e4m3, f32 = torch.float8_e4m3fn, torch.float32
    kb, nb = -(-K // _BLOCK), -(-N // _BLOCK)
    s = {"case": case}
    if kind == "rows":
        x = normal(R, K) * torch.exp(torch.randn((R, 1), device="cuda", generator=gen)).to(dtype)  # rows of different size
        return dict(s, x=x, q=empty(R, K, dtype=e4m3), scales=empty(R, kb, dtype=f32))
    if kind == "weights":
        w = torch.stack([normal(N, K, std=K ** -0.5) for _ in range(E)])
        return dict(s, w=w, q=empty(E, N, K, dtype=e4m3), scales=empty(E, nb, kb, dtype=f32),
                    q_t=empty(E, K, N, dtype=e4m3), scales_t=empty(E, kb, nb, dtype=f32))
    s["plan"] = _offsets(case, seed)
    s["offsets"] = torch.tensor(s["plan"], dtype=torch.int32, device="cuda")
    if kind == "fp8":
        x = _rows_to_e4m3(torch.randn((R, K), device="cuda", generator=gen))
        w = [_tiles_to_e4m3(torch.randn((N, K), device="cuda", generator=gen).mul_(K ** -0.5)) for _ in range(E)]
        return dict(s, xq=x[0], xs=x[1], wq=torch.stack([q for q, _ in w]), ws=torch.stack([t for _, t in w]), y=empty(R, N))
    s["w"] = torch.stack([normal(N, K, std=K ** -0.5) for _ in range(E)])
    s["x"] = normal(R, K)
    if kind == "product":
        return dict(s, y=empty(R, N))
    return dict(s, dy=normal(R, N), dx=empty(R, K), dw=empty(E, N, K, dtype=_DTYPES[case["dw"]]))


def _scale_of(amax):
    scale = amax.clamp_min(_LEAST_AMAX) / torch.full_like(amax, _E4M3_MAX)   # (by a number, it would be multiplied by 1 / 448)
    return torch.where(torch.isfinite(scale), scale, math.nan)


def _rows_to_e4m3(x):
    R, K = x.shape
    pad = -K % _BLOCK
    blocks = torch.nn.functional.pad(x.float(), (0, pad)).view(R, -1, _BLOCK)
    scale = _scale_of(blocks.abs().amax(2))
    return (blocks / scale[:, :, None]).view(R, K + pad)[:, :K].to(torch.float8_e4m3fn), scale


def _tiles_to_e4m3(w):
    N, K = w.shape
    tiles = torch.nn.functional.pad(w.float(), (0, -K % _BLOCK, 0, -N % _BLOCK))
    tiles = tiles.view(-(-N // _BLOCK), _BLOCK, -(-K // _BLOCK), _BLOCK)
    scale = _scale_of(tiles.abs().amax(3).amax(1))
    q = (tiles / scale[:, None, :, None]).view(tiles.shape[0] * _BLOCK, tiles.shape[2] * _BLOCK)[:N, :K]
    return q.to(torch.float8_e4m3fn).contiguous(), scale


def _per_expert(state):
    """(expert, its first row, the row behind its last) of every expert that has rows.  One product for each of them is the
    shortest plain form: rows padded to one batched product would compute several times as much under a skewed routing."""
    plan = state["plan"]
    return [(e, a, b) for e, (a, b) in enumerate(zip(plan, plan[1:])) if b > a]


def _plain(state):
    case = state["case"]
    kind, dtype = case["kind"], _DTYPES[case["dtype"]]
    if kind == "rows":
        return _rows_to_e4m3(state["x"])
    if kind == "weights":
        for e in range(case["experts"]):
            q, scale = _tiles_to_e4m3(state["w"][e])
            state["q"][e], state["scales"][e], state["q_t"][e], state["scales_t"][e] = q, scale, q.t(), scale.t()
        return state["q"], state["scales"], state["q_t"], state["scales_t"]
    if kind == "product":
        for e, a, b in _per_expert(state):
            state["y"][a:b] = state["x"][a:b].float() @ state["w"][e].float().t()
        return state["y"]
    if kind == "fp8":
        N, K = case["n"], case["k"]
        x = state["xq"].float() * state["xs"].repeat_interleave(_BLOCK, 1)[:, :K]
        for e, a, b in _per_expert(state):
            scale = state["ws"][e].repeat_interleave(_BLOCK, 0)[:N].repeat_interleave(_BLOCK, 1)[:, :K]
            state["y"][a:b] = x[a:b] @ (state["wq"][e].float() * scale).t()
        return state["y"]
    if len(_per_expert(state)) < case["experts"]:
        state["dw"].zero_()
    for e, a, b in _per_expert(state):
        dy = state["dy"][a:b].float()
        state["dx"][a:b] = dy @ state["w"][e].float()
        state["dw"][e] = dy.t() @ state["x"][a:b].float()
    return state["dx"], state["dw"]


def run(state):
    if not own:
        return _plain(state)
    from paper_2501_10375_amd import products

    case, s = state["case"], state
    kind = case["kind"]
    if kind == "rows":
        products.moe_quantize_rows_fp8(s["x"], s["q"], s["scales"])
        return s["q"], s["scales"]
    if kind == "weights":
        products.moe_quantize_weights_fp8(s["w"], s["q"], s["scales"], s["q_t"], s["scales_t"])
        return s["q"], s["scales"], s["q_t"], s["scales_t"]
    if "workspace" not in s:   # scratch that a program keeps for its calls
        shape = products.make_product(case["experts"], case["n"], case["k"], _DTYPES[case["dtype"]])
        s["workspace"] = products.alloc_workspace(shape, case["rows"])
    if kind == "product":
        products.moe_grouped_product(s["x"], s["offsets"], s["w"], s["y"], s["workspace"])
        return s["y"]
    if kind == "fp8":
        products.moe_grouped_product_fp8(s["xq"], s["xs"], s["offsets"], s["wq"], s["ws"], s["y"], s["workspace"])
        return s["y"]
    products.moe_grouped_product_dgrad(s["dy"], s["offsets"], s["w"], s["dx"], s["workspace"])
    products.moe_grouped_product_wgrad(s["dy"], s["x"], s["offsets"], s["dw"], False, s["workspace"])
    return s["dx"], s["dw"]


def work(case):
    """Bytes and operations of one pass: every input that the rows need read once, every output written once.  Where there are
    fewer rows than experts, at most one expert a row has its weights read."""
    E, N, K, R = case["experts"], case["n"], case["k"], case["rows"]
    size = 4 if case["dtype"] == "f32" else 2
    used, kb, nb = min(E, R), -(-K // _BLOCK), -(-N // _BLOCK)
    if case["kind"] == "rows":
        return {"bytes": R * K * (size + 1) + 4 * R * kb, "flops": 0}
    if case["kind"] == "weights":
        return {"bytes": E * N * K * (size + 2) + 8 * E * nb * kb, "flops": 0}
    if case["kind"] == "product":
        return {"bytes": size * (R * (N + K) + used * N * K) + 4 * (E + 1), "flops": 2 * R * N * K}
    if case["kind"] == "fp8":
        return {"bytes": R * K + 4 * R * kb + used * (N * K + 4 * nb * kb) + size * R * N + 4 * (E + 1), "flops": 2 * R * N * K}
    dw = 4 if case["dw"] == "f32" else 2
    return {"bytes": size * (2 * R * (N + K) + used * N * K) + dw * E * N * K + 4 * (E + 1), "flops": 4 * R * N * K}


def _nearest_e4m3(v):
    """float64 -> the nearest value of e4m3 (ties to even), as float64.  Steps of 2^-3 of the leading power of two, 2^-9 below 2^-6."""
    _, exponent = torch.frexp(v)
    step = ((exponent.long() - 1).clamp_min(-6) - 3 + 1023).bitwise_left_shift(52).view(torch.float64)   # (pow(2, n) may be off)
    return torch.round(v / step) * step


def exact(case, seed):
    """What run() returns, in 64 bits: sums over the definition, scales and quotients rounded to fp32 as the definition says."""
    s = prepare(case, seed)
    E, N, K, kind = case["experts"], case["n"], case["k"], case["kind"]
    to32 = lambda v: v.to(torch.float32).double()  # noqa: E731

    def quantised(v, rows, cols):
        """A matrix in blocks of rows x cols: values of e4m3 and scales."""
        at_r = torch.arange(v.shape[0], device=v.device) // rows
        at_k = torch.arange(v.shape[1], device=v.device) // cols
        at = at_r[:, None] * (-(-v.shape[1] // cols)) + at_k[None, :]
        amax = torch.zeros(int(at.max()) + 1, dtype=torch.float64, device=v.device)
        amax.scatter_reduce_(0, at.reshape(-1), v.abs().reshape(-1), "amax")
        scale = to32(torch.clamp(amax, min=_LEAST_AMAX) / _E4M3_MAX)
        return _nearest_e4m3(to32(v / scale[at])), scale.view(-1, -(-v.shape[1] // cols))

    if kind == "rows":
        parts = [quantised(x.double(), 1, _BLOCK) for x in s["x"].split(2048)]
        return torch.cat([q.float() for q, _ in parts]), torch.cat([t for _, t in parts])
    if kind == "weights":
        parts = [quantised(w.double(), _BLOCK, _BLOCK) for w in s["w"]]
        q, scale = torch.stack([q.float() for q, _ in parts]), torch.stack([t for _, t in parts])
        return q, scale, q.transpose(1, 2).contiguous(), scale.transpose(1, 2).contiguous()
    spans = [slice(a, b) for a, b in zip(s["plan"], s["plan"][1:])]
    if kind == "product":
        return torch.cat([s["x"][r].double() @ s["w"][e].double().mT for e, r in enumerate(spans)])
    if kind == "fp8":
        out = []
        for e, r in enumerate(spans):
            y = torch.zeros((r.stop - r.start, N), dtype=torch.float64, device="cuda")
            for b in range(-(-K // _BLOCK)):
                k = slice(b * _BLOCK, min(K, (b + 1) * _BLOCK))
                inner = s["xq"][r, k].double() @ s["wq"][e][:, k].double().mT
                scale = s["xs"][r, b].double()[:, None] * s["ws"][e][:, b].double().repeat_interleave(_BLOCK)[None, :N]
                y += inner * scale
            out.append(y)
        return torch.cat(out)
    dx = torch.cat([s["dy"][r].double() @ s["w"][e].double() for e, r in enumerate(spans)])
    dw = torch.stack([s["dy"][r].double().mT @ s["x"][r].double() for r in spans])
    return dx, dw
