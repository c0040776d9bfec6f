"""Workloads of the training operators next to the slim layers: layer normalisation over the channels of a pixel
(forward, and backward with the gradients of its weight and bias) and the orthogonalised update of a filter matrix
(Newton-Schulz products, alone and as a whole optimiser step on float32 master weights).

Every workload can be computed two ways: with elementary torch operations in float32, rounded once at the end
(``own`` false), or with the library's own entry points (``own`` true).  ``exact`` gives the same outputs from the
definitions in float64.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS_LN = 1e-5
EPS_NS = 1e-7
NS_STEPS = 5
NS_COEF = (3.4445, -4.7750, 2.0315)       # the quintic's usual coefficients
MOMENTUM, DECAY = 0.95, 0.01


def listed():
    return [
        # the last module's 7 x 7 plane of one image: the call whose time is its latency
        {"name": "ln_49x1024", "op": "layernorm", "pixels": 49, "channels": 1024, "x": "bf16", "y": "bf16", "slice": False},
        # an ordinary ragged layer: one branch of a concatenated module output, an odd number of channels
        {"name": "ln_50176x333_slice", "op": "layernorm", "pixels": 50176, "channels": 333, "x": "bf16", "y": "bf16", "slice": True},
        # inception 3a's output at batch 256
        {"name": "ln_200704x256", "op": "layernorm", "pixels": 200704, "channels": 256, "x": "bf16", "y": "bf16", "slice": False},
        # the backward pass of the same single image, of a float32 stream with bfloat16 gradients, and at batch 256
        {"name": "ln_bwd_49x1024", "op": "layernorm_bwd", "pixels": 49, "channels": 1024, "x": "bf16", "y": "bf16", "slice": False},
        {"name": "ln_bwd_12544x2048_f32", "op": "layernorm_bwd", "pixels": 12544, "channels": 2048, "x": "f32", "y": "bf16", "slice": False},
        {"name": "ln_bwd_200704x256", "op": "layernorm_bwd", "pixels": 200704, "channels": 256, "x": "bf16", "y": "bf16", "slice": False},
        # a 1 x 1 layer that widens 512 channels to 2048: more rows than columns
        {"name": "ns_2048x512", "op": "orthogonalise", "batch": 1, "rows": 2048, "cols": 512, "g": "bf16"},
        # a classifier of 1000 classes on 2048 features: 1000 is no multiple of a tile
        {"name": "ns_1000x2048", "op": "orthogonalise", "batch": 1, "rows": 1000, "cols": 2048, "g": "f32"},
        # the largest fully connected layer of the networks here
        {"name": "ns_4096x9216", "op": "orthogonalise", "batch": 1, "rows": 4096, "cols": 9216, "g": "f32"},
        # the 7 x 7 stem on three channels: 147 columns, the smallest step
        {"name": "muon_64x147", "op": "muon_update", "batch": 1, "rows": 64, "cols": 147, "nesterov": True, "lr": 0.002},
        # six 3 x 3 layers of 256 channels (one residual stage), updated in one call
        {"name": "muon_6x256x2304", "op": "muon_update", "batch": 6, "rows": 256, "cols": 2304, "nesterov": True, "lr": 0.001},
        # a merged 5 x 5 layer of inception 4e: 512 filters of 25 x 528 values
        {"name": "muon_512x13200", "op": "muon_update", "batch": 1, "rows": 512, "cols": 13200, "nesterov": False, "lr": 0.0005},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["layernorm", "layernorm_bwd", "orthogonalise", "muon_update"])
    if op.startswith("layernorm"):
        channels = _log_uniform(rng, 16, 8192)
        if rng.random() < 0.6:
            channels = max(16, channels // 8 * 8)
        pixels = _log_uniform(rng, 1, min(200704, 200704 * 256 // channels))
        return {"op": op, "pixels": pixels, "channels": channels, "x": rng.choice(["bf16", "bf16", "f32"]),
                "y": rng.choice(["bf16", "bf16", "f32"]), "slice": rng.random() < 0.25}
    while True:
        batch = rng.choice([1, 1, 1, 2, 3, 6, 9])
        rows, cols = _log_uniform(rng, 16, 4096), _log_uniform(rng, 16, 20800)
        if rng.random() < 0.6:
            rows, cols = max(16, rows // 8 * 8), max(16, cols // 8 * 8)
        n, m = min(rows, cols), max(rows, cols)
        if batch * n * n * (3 * m + n) <= 4096 * 4096 * (3 * 9216 + 4096) and batch * rows * cols <= 4096 * 9216:
            break
    case = {"op": op, "batch": batch, "rows": rows, "cols": cols}
    if op == "orthogonalise":
        case["g"] = rng.choice(["bf16", "f32"])
    else:
        case["nesterov"] = rng.random() < 0.7
        case["lr"] = rng.choice([0.0005, 0.001, 0.002])
    return case


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    if case["op"] == "layernorm":
        n = case["pixels"] * case["channels"]
        return {"bytes": n * (_size(case["x"]) + _size(case["y"])) + 8 * case["pixels"] + 8 * case["channels"], "flops": 7 * n}
    if case["op"] == "layernorm_bwd":
        n = case["pixels"] * case["channels"]
        return {"bytes": n * (2 * _size(case["x"]) + _size(case["y"])) + 8 * case["pixels"] + 12 * case["channels"], "flops": 14 * n}
    n, m = sorted((case["rows"], case["cols"]))
    # per step a symmetric n x n product over m (half of it), a symmetric one over n, and one n x n by n x m
    flops = case["batch"] * NS_STEPS * (n * n * m + n * n * n + 2 * n * n * m)
    size = case["batch"] * n * m
    if case["op"] == "orthogonalise":
        return {"bytes": size * (_size(case["g"]) + 2), "flops": flops}
    return {"bytes": size * (4 + 8 + 8 + 2), "flops": flops}          # g read, v and w read and written, the bfloat16 copy written


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(g, pixels, channels, dtype, wide):
    """A [pixels, channels] activation: per-channel offsets and a few strong channels, as feature maps have; with
    `wide` a channel slice of a wider tensor."""
    ld = channels + (channels // 2 + 8) // 8 * 8 if wide else channels
    full = torch.randn((pixels, ld), generator=g, device="cuda")
    full *= 0.2 + torch.rand((ld,), generator=g, device="cuda") ** 4 * 5
    full += 0.5 * torch.randn((ld,), generator=g, device="cuda")
    return full.to(dtype)[:, ld - channels:]


def _gradient(g, batch, rows, cols):
    """A gradient matrix: a few strong directions over noise."""
    r = min(16, rows, cols)
    strong = torch.randn((batch, rows, r), generator=g, device="cuda") @ torch.randn((batch, r, cols), generator=g, device="cuda")
    return (strong * (0.3 / math.sqrt(r)) + torch.randn((batch, rows, cols), generator=g, device="cuda")) * 1e-3


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["op"].startswith("layernorm"):
        M, C = case["pixels"], case["channels"]
        xt, yt = DTYPES[case["x"]], DTYPES[case["y"]]
        s["x"] = _rows(g, M, C, xt, case["slice"])
        s["gamma"] = 1 + 0.1 * torch.randn((C,), generator=g, device="cuda")
        s["beta"] = 0.1 * torch.randn((C,), generator=g, device="cuda")
        if case["op"] == "layernorm_bwd":
            s["dy"] = (1e-2 * torch.randn((M, C), generator=g, device="cuda")).to(yt)
            x = s["x"].float()                        # the statistics that the forward pass kept
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + EPS_LN)
        if own:
            import paper_1708_04728_b200 as dr
            s["dr"] = dr
            s["flags"] = (dr.DR_LN_X_F32 if case["x"] == "f32" else 0) | (dr.DR_LN_Y_F32 if case["y"] == "f32" else 0)
            if case["op"] == "layernorm":
                s["out"] = (torch.empty((M, C), dtype=yt, device="cuda"), torch.empty((M,), device="cuda"), torch.empty((M,), device="cuda"))
            else:
                s["out"] = (torch.empty((M, C), dtype=xt, device="cuda"), torch.empty((C,), device="cuda"), torch.empty((C,), device="cuda"))
                s["ws"] = torch.empty(dr.dr_layernorm_bwd_workspace_bytes(M, C), dtype=torch.uint8, device="cuda")
        return s
    B, R, K = case["batch"], case["rows"], case["cols"]
    if case["op"] == "orthogonalise":
        s["g"] = _gradient(g, B, R, K).to(DTYPES[case["g"]])
    else:
        s["g"] = _gradient(g, B, R, K)
        s["v"] = 3 * _gradient(g, B, R, K)
        s["w"] = math.sqrt(2 / K) * torch.randn((B, R, K), generator=g, device="cuda")     # He initialisation
    if own:
        import paper_1708_04728_b200 as dr
        s["dr"] = dr
        s["ws"] = torch.empty(dr.dr_orthogonalise_workspace_bytes(B, R, K), dtype=torch.uint8, device="cuda")
        s["bf16"] = torch.empty((B, R, K), dtype=torch.bfloat16, device="cuda")
    return s


def _newton_schulz(u):
    """X <- X / (|X| + eps), then per step A = X X^T, X <- a X + (b A + c A A) X; on the transpose where that has fewer rows."""
    a, b, c = NS_COEF
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS_NS)
    for _ in range(NS_STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2) if tall else x


def _plain(s):
    case = s["case"]
    if case["op"] == "layernorm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS_LN)
        return (d * rstd * s["gamma"] + s["beta"]).to(DTYPES[case["y"]]), mean[:, 0], rstd[:, 0]
    if case["op"] == "layernorm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xhat = (s["x"].float() - s["mean"][:, None]) * rstd
        t = dy * s["gamma"]
        dx = rstd * (t - t.mean(1, keepdim=True) - xhat * (t * xhat).mean(1, keepdim=True))
        return dx.to(DTYPES[case["x"]]), (dy * xhat).sum(0), dy.sum(0)
    if case["op"] == "orthogonalise":
        return _newton_schulz(s["g"].float()).to(torch.bfloat16).contiguous()
    s["v"].mul_(MOMENTUM).add_(s["g"])
    u = s["g"] + MOMENTUM * s["v"] if case["nesterov"] else s["v"]
    scale = math.sqrt(max(1.0, case["rows"] / case["cols"]))
    s["w"].mul_(1 - case["lr"] * DECAY).sub_(_newton_schulz(u), alpha=case["lr"] * scale)
    return s["w"], s["v"], s["w"].to(torch.bfloat16)


def run(state):
    s = state
    if not own:
        return _plain(s)
    case, dr = s["case"], s["dr"]
    if case["op"] == "layernorm":
        y, mean, rstd = s["out"]
        dr.dr_layernorm(case["pixels"], case["channels"], s["x"], s["x"].stride(0), s["gamma"], s["beta"], EPS_LN, y, case["channels"],
                        mean, rstd, s["flags"])
        return y, mean, rstd
    if case["op"] == "layernorm_bwd":
        dx, dgamma, dbeta = s["out"]
        dr.dr_layernorm_bwd(case["pixels"], case["channels"], s["dy"], case["channels"], s["x"], s["x"].stride(0), s["gamma"], s["mean"], s["rstd"],
                            dx, case["channels"], dgamma, dbeta, s["ws"], s["ws"].numel(), s["flags"])
        return dx, dgamma, dbeta
    B, R, K = case["batch"], case["rows"], case["cols"]
    if case["op"] == "orthogonalise":
        dr.dr_orthogonalise(B, R, K, s["g"], NS_STEPS, None, EPS_NS, s["bf16"], s["ws"], s["ws"].numel(),
                            dr.DR_NS_G_F32 if case["g"] == "f32" else 0)
        return s["bf16"]
    dr.dr_muon_update(B, R, K, s["w"], s["v"], s["g"], case["lr"], MOMENTUM, DECAY, case["nesterov"], NS_STEPS, None, EPS_NS, s["bf16"],
                      s["ws"], s["ws"].numel())
    return s["w"], s["v"], s["bf16"]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "layernorm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS_LN)
        return torch.addcmul(s["beta"].double(), (x - mean[:, None]) * rstd[:, None], s["gamma"].double()), mean, rstd
    if case["op"] == "layernorm_bwd":
        # the gradients of y = gamma * xhat + beta with the statistics the forward pass kept
        x, dy, gamma = s["x"].double(), s["dy"].double(), s["gamma"].double()
        rstd = s["rstd"].double()[:, None]
        xhat = (x - s["mean"].double()[:, None]) * rstd
        C = x.shape[1]
        s1 = dy @ gamma / C
        s2 = torch.einsum("mc,mc,c->m", dy, xhat, gamma) / C
        dx = (dy * gamma - s1[:, None] - xhat * s2[:, None]) * rstd
        return dx, torch.einsum("mc,mc->c", dy, xhat), torch.einsum("mc->c", dy)
    a, b, c = NS_COEF

    def polynomial(u):
        # an odd polynomial of the matrix: u p(u^T u) = p(u u^T) u, so the smaller of the two Gram matrices serves
        x = u / (torch.linalg.matrix_norm(u, keepdim=True) + EPS_NS)
        eye = torch.eye(min(u.shape[1:]), dtype=torch.float64, device="cuda")
        for _ in range(NS_STEPS):
            if u.shape[1] <= u.shape[2]:
                gram = torch.bmm(x, x.mT)
                x = torch.bmm(a * eye + b * gram + c * torch.bmm(gram, gram), x)
            else:
                gram = torch.bmm(x.mT, x)
                x = torch.bmm(x, a * eye + b * gram + c * torch.bmm(gram, gram))
        return x

    if case["op"] == "orthogonalise":
        return polynomial(s["g"].double())
    grad, v, w = s["g"].double(), s["v"].double(), s["w"].double()
    v = MOMENTUM * v + grad
    o = polynomial(grad + MOMENTUM * v if case["nesterov"] else v)
    w = w - case["lr"] * (math.sqrt(max(1.0, case["rows"] / case["cols"])) * o + DECAY * w)
    return w, v, w
