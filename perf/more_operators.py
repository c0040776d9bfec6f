"""Workloads of the operators that re-learn and serve variants of a slim layer: dropout from a counter-based generator
(whose mask is never stored), a 1 x 1 (or fully connected) layer with the low-rank adapters of many requests beside its
shared filters, and that layer's gradients for its input and for the adapters, with dropout in front of them or without.

Every workload can be computed two ways: with elementary torch operations in float32, rounded once at the end
(``own`` false), or with the library's own entry points (``own`` true).  ``exact`` gives the same outputs from the
definitions in float64.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # a training batch's pooled features in front of the classifier, 40 % dropped: the call whose time is its latency
        {"name": "drop_32x1024", "op": "dropout", "rows": 32, "channels": 1024, "x": "bf16", "y": "bf16", "p": 0.4, "residual": False, "slice": False},
        # a slice of a concatenated module output with an odd number of channels, float32
        {"name": "drop_50176x333_f32_slice", "op": "dropout", "rows": 50176, "channels": 333, "x": "f32", "y": "f32", "p": 0.1, "residual": False, "slice": True},
        # a residual branch at batch 256, dropped as it is added
        {"name": "drop_200704x256_residual", "op": "dropout", "rows": 200704, "channels": 256, "x": "bf16", "y": "bf16", "p": 0.1, "residual": True, "slice": False},
        # the classifier of one image for one request: latency again
        {"name": "adapter_1x1024x1000_r8", "op": "adapter", "rows": 1, "cin": 1024, "cout": 1000, "rank": 8, "adapters": 4, "segments": 1,
         "ragged": False, "p": 0.0, "relu": False, "y": "f32", "slice": False},
        # 32 requests of 32 variants at once through a 4096 x 4096 layer: the filters are read once for all of them
        {"name": "adapter_32x4096x4096_r16", "op": "adapter", "rows": 32, "cin": 4096, "cout": 4096, "rank": 16, "adapters": 32, "segments": 32,
         "ragged": False, "p": 0.0, "relu": True, "y": "bf16", "slice": False},
        # requests of different lengths through a 528-channel reducer, an odd rank, some requests without an adapter, rows of none
        {"name": "adapter_7001x528x160_r12", "op": "adapter", "rows": 7001, "cin": 528, "cout": 160, "rank": 12, "adapters": 9, "segments": 37,
         "ragged": True, "p": 0.0, "relu": True, "y": "bf16", "slice": True},
        # re-learning a residual expansion at 56 x 56 and batch 64, with dropout in front of the adapter: bound by memory
        {"name": "adapter_200704x64x256_r8_drop", "op": "adapter", "rows": 200704, "cin": 64, "cout": 256, "rank": 8, "adapters": 4, "segments": 64,
         "ragged": False, "p": 0.1, "relu": True, "y": "bf16", "slice": False},
        # many rows through a fully connected layer: bound by the products
        {"name": "adapter_16384x4096x4096_r64", "op": "adapter", "rows": 16384, "cin": 4096, "cout": 4096, "rank": 64, "adapters": 8, "segments": 16,
         "ragged": False, "p": 0.0, "relu": False, "y": "bf16", "slice": False},
        # the gradients of one 7 x 7 image of one request
        {"name": "adapter_bwd_49x832x384_r8", "op": "adapter_bwd", "rows": 49, "cin": 832, "cout": 384, "rank": 8, "adapters": 1, "segments": 1,
         "ragged": False, "p": 0.0, "slice": False},
        # a residual reducer at 7 x 7 and batch 256, images of eight variants, with dropout
        {"name": "adapter_bwd_12544x2048x512_r16_drop", "op": "adapter_bwd", "rows": 12544, "cin": 2048, "cout": 512, "rank": 16, "adapters": 8,
         "segments": 256, "ragged": False, "p": 0.1, "slice": False},
        # the gradients of the large fully connected layer
        {"name": "adapter_bwd_16384x4096x4096_r64", "op": "adapter_bwd", "rows": 16384, "cin": 4096, "cout": 4096, "rank": 64, "adapters": 8,
         "segments": 16, "ragged": False, "p": 0.0, "slice": False},
    ]


LARGEST = 16384 * 4096 * 4096          # rows x cin x cout of the largest listed case
ELEMENTS = 200704 * 256


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dropout", "adapter", "adapter", "adapter_bwd", "adapter_bwd"])
    if op == "dropout":
        channels = _log_uniform(rng, 16, 9216)
        if rng.random() < 0.6:
            channels = max(16, channels // 8 * 8)
        return {"op": op, "rows": _log_uniform(rng, 1, max(1, ELEMENTS // channels)), "channels": channels, "x": rng.choice(["bf16", "bf16", "f32"]),
                "y": rng.choice(["bf16", "bf16", "f32"]), "p": rng.choice([0.1, 0.25, 0.4, 0.5, 0.7]), "residual": rng.random() < 0.4,
                "slice": rng.random() < 0.25}
    while True:
        cin, cout, rows = _log_uniform(rng, 48, 9216), _log_uniform(rng, 48, 4096), _log_uniform(rng, 1, 200704)
        if rng.random() < 0.75:
            cin = cin // 8 * 8
        if rng.random() < 0.75:
            cout = cout // 8 * 8
        rank = rng.choice([4, 8, 8, 12, 16, 16, 32, 64, 5])
        adapters = _log_uniform(rng, 1, 64)
        if rows * cin * cout <= LARGEST and rows * max(cin, cout) <= 16384 * 4096 and adapters * (cin + cout) * rank <= 64 * 8192 * 16:
            break
    # up to a few hundred requests; one row each where rows are few (single tokens), longer ones elsewhere
    segments = rows if rows <= 128 and rng.random() < 0.6 else min(rows, _log_uniform(rng, 1, 256))
    case = {"op": op, "rows": rows, "cin": cin, "cout": cout, "rank": rank, "adapters": adapters, "segments": segments,
            "ragged": rng.random() < 0.5, "p": rng.choice([0.0, 0.0, 0.1, 0.25]), "slice": rng.random() < 0.2}
    if op == "adapter":
        case["relu"] = rng.random() < 0.5
        case["y"] = rng.choice(["bf16", "bf16", "f32"])
    return case


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    if case["op"] == "dropout":
        n = case["rows"] * case["channels"]
        return {"bytes": n * (_size(case["x"]) + _size(case["y"]) * (2 if case["residual"] else 1)), "flops": 2 * n}
    M, K, N, R = case["rows"], case["cin"], case["cout"], case["rank"]
    used = min(case["adapters"], case["segments"])
    if case["op"] == "adapter":
        return {"bytes": 2 * (M * K + N * K + used * R * (K + N)) + M * N * _size(case["y"]), "flops": 2 * M * (N * K + R * (K + N))}
    return {"bytes": 2 * (2 * M * K + M * N + N * K + used * R * (K + N)) + 4 * (M * R + case["adapters"] * R * (K + N)),
            "flops": 2 * M * (N * K + 2 * R * (K + N))}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _wider(t, wide):
    """The same values as a channel slice of a wider tensor."""
    if not wide:
        return t
    full = torch.full((t.shape[0], t.shape[1] + 24), 3.0, dtype=t.dtype, device="cuda")
    full[:, 8:8 + t.shape[1]] = t
    return full[:, 8:8 + t.shape[1]]


def _features(g, rows, channels):
    """A feature map: ReLU of normal values, channels of different strength."""
    x = torch.randn((rows, channels), generator=g, device="cuda").relu_()
    return x.mul_(0.3 + torch.rand((channels,), generator=g, device="cuda") ** 3 * 2)


def _requests(case, seed):
    """Row offsets and adapter of every request (host lists).  Ragged: lengths of all sizes, empty ones among them, one request in ten
    without an adapter, and rows behind the last request where there are enough."""
    rng = np.random.default_rng(seed)
    M, S, A = case["rows"], case["segments"], case["adapters"]
    ids = (np.arange(S) + int(rng.integers(A))) % A
    rng.shuffle(ids)
    if not case["ragged"]:
        starts = [M * i // S for i in range(S + 1)]
    else:
        total = M - M // 64
        cuts = np.sort(np.concatenate([[0, total], rng.integers(0, total + 1, S - 1)]))
        starts = [int(c) for c in cuts]
        ids[rng.random(S) < 0.1] = -1
    return starts, [int(i) for i in ids]


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": case, "seed": 1000 + seed, "offset": 7 * seed + 3}
    if case["op"] == "dropout":
        M, C = case["rows"], case["channels"]
        s["x"] = _wider(_features(g, M, C).to(DTYPES[case["x"]]), case["slice"])
        s["residual"] = _wider(torch.randn((M, C), generator=g, device="cuda").to(DTYPES[case["y"]]), case["slice"]) if case["residual"] else None
        if own:
            import paper_1708_04728_b200 as dr
            s["dr"] = dr
            s["flags"] = (dr.DR_DROP_X_F32 if case["x"] == "f32" else 0) | (dr.DR_DROP_Y_F32 if case["y"] == "f32" else 0)
            s["y"] = torch.empty((M, C), dtype=DTYPES[case["y"]], device="cuda")
        return s
    M, K, N, R, A = case["rows"], case["cin"], case["cout"], case["rank"], case["adapters"]
    s["x"] = _wider(_features(g, M, K).to(torch.bfloat16), case["slice"])
    s["w"] = (math.sqrt(2 / K) * torch.randn((N, K), generator=g, device="cuda")).to(torch.bfloat16)
    s["a"] = (math.sqrt(1 / K) * torch.randn((A, R, K), generator=g, device="cuda")).to(torch.bfloat16)
    s["b"] = (0.2 * math.sqrt(1 / R) * torch.randn((A, N, R), generator=g, device="cuda")).to(torch.bfloat16)
    s["scale"] = 0.5 + torch.rand((A,), generator=g, device="cuda")
    s["starts"], s["ids"] = _requests(case, seed)
    s["row_start"] = torch.tensor(s["starts"], dtype=torch.int32, device="cuda")
    s["adapter"] = torch.tensor(s["ids"], dtype=torch.int32, device="cuda")
    if case["op"] == "adapter":
        s["bias"] = 0.1 * torch.randn((N,), generator=g, device="cuda")
        s["y"] = _wider(torch.zeros((M, N), dtype=DTYPES[case["y"]], device="cuda"), case["slice"])
        s["t"] = torch.zeros((M, R), device="cuda") if case["p"] else None        # kept for the backward pass where the layer is trained
    else:
        s["dy"] = (1e-2 * torch.randn((M, N), generator=g, device="cuda")).to(torch.bfloat16)
        # what the forward pass kept: each row's product with its adapter's first factor
        s["t"] = torch.zeros((M, R), device="cuda")
        x = _dropped(s["x"].float(), s)
        for a, rows in _groups(s):
            s["t"][rows] = x[rows] @ s["a"][a].float().T
        s["dx"] = _wider(torch.zeros((M, K), dtype=torch.bfloat16, device="cuda"), case["slice"])
    if own:
        import paper_1708_04728_b200 as dr
        s["dr"] = dr
        flags = 0
        if case["op"] == "adapter":
            flags = dr.DR_BIAS | (dr.DR_RELU if case["relu"] else 0) | (dr.DR_OUT_F32 if case["y"] == "f32" else 0)
        s["desc"] = dr.dr_adapter_desc(Cin=K, Cout=N, rank=R, adapters=A, flags=flags, drop_p=case["p"], drop_seed=s["seed"], drop_offset=s["offset"])
        if case["op"] == "adapter":
            n = dr.dr_adapter_workspace_bytes(s["desc"], M, s["x"].stride(0))
        else:
            n = dr.dr_adapter_bwd_workspace_bytes(s["desc"], M, s["x"].stride(0), s["dy"].stride(0))
            s["da"], s["db"] = torch.empty((A, R, K), device="cuda"), torch.empty((A, N, R), device="cuda")
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


def _words(index, seed, offset):
    """Philox4x32-10 of the counters (index, offset) under the key `seed`: four 32-bit words for each index, as int64."""
    low = 0xFFFFFFFF

    def product(m, v):                     # high and low word of a 32 x 32 bit product, in int64 without overflow
        p0, p1 = v * (m & 0xFFFF), v * (m >> 16)
        p1 = p1 + (p0 >> 16)
        return p1 >> 16, ((p1 & 0xFFFF) << 16) | (p0 & 0xFFFF)

    c = [index & low, index >> 32, torch.full_like(index, offset & low), torch.full_like(index, offset >> 32)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        h0, l0 = product(0xD2511F53, c[0])
        h1, l1 = product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _threshold(p):
    return int(math.floor(p * 65536 + 0.5))


def _dropped(x, s):
    """x with dropped elements zero and the others divided by the share that is kept.  Element e of a row-major [rows, channels] takes 16 bits of
    the generator: word (e mod 8) / 2 of counter e / 8, its low half first; it is dropped where they are below p 2^16."""
    if not s["case"]["p"]:
        return x
    n = x.numel()
    t = _threshold(s["case"]["p"])
    words = _words(torch.arange((n + 7) // 8, device="cuda"), s["seed"], s["offset"])
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], 1).reshape(-1)[:n].reshape(x.shape)
    return x * (halves >= t) * (65536 / (65536 - t))


def _groups(s):
    """(adapter, its rows) for each adapter in use: a slice, or an index tensor."""
    rows = {}
    for i, a in enumerate(s["ids"]):
        if a >= 0 and s["starts"][i + 1] > s["starts"][i]:
            rows.setdefault(a, []).append((s["starts"][i], s["starts"][i + 1]))
    for a, parts in sorted(rows.items()):
        if len(parts) == 1:
            yield a, slice(*parts[0])
        else:
            yield a, torch.cat([torch.arange(u, v, device="cuda") for u, v in parts])


def _plain(s):
    case = s["case"]
    if case["op"] == "dropout":
        y = _dropped(s["x"].float(), s)
        if s["residual"] is not None:
            y = s["residual"].float() + y
        return y.to(DTYPES[case["y"]])
    x, w = s["x"].float(), s["w"].float()
    first, last = s["starts"][0], s["starts"][-1]              # rows of no request are left as they were
    if case["op"] == "adapter":
        y = x @ w.T + s["bias"]
        xd = _dropped(x, s)
        t = torch.zeros((case["rows"], case["rank"]), device="cuda")
        for a, rows in _groups(s):
            t[rows] = xd[rows] @ s["a"][a].float().T
            y[rows] += (t[rows] @ s["b"][a].float().T) * s["scale"][a]
        if case["relu"]:
            y = torch.clamp(y, min=0)
        s["y"][first:last] = y[first:last].to(s["y"].dtype)
        if s["t"] is None:
            return s["y"]
        s["t"][first:last] = t[first:last]
        return s["y"], s["t"]
    dy = s["dy"].float()
    dx = dy @ w
    xd = _dropped(x, s)
    part = torch.zeros_like(dx)
    da, db = torch.zeros(s["a"].shape, device="cuda"), torch.zeros(s["b"].shape, device="cuda")
    for a, rows in _groups(s):
        u = (dy[rows] @ s["b"][a].float()) * s["scale"][a]
        part[rows] = u @ s["a"][a].float()
        da[a] = u.T @ xd[rows]
        db[a] = (dy[rows].T @ s["t"][rows]) * s["scale"][a]
    dx = dx + _dropped(part, s)
    s["dx"][first:last] = dx[first:last].to(torch.bfloat16)
    return s["dx"], da, db


def run(state):
    s = state
    if not own:
        return _plain(s)
    case, dr = s["case"], s["dr"]
    if case["op"] == "dropout":
        r = s["residual"]
        dr.dr_dropout(case["rows"], case["channels"], s["x"], s["x"].stride(0), r, r.stride(0) if r is not None else 0, s["y"], case["channels"],
                      case["p"], s["seed"], s["offset"], None, s["flags"])
        return s["y"]
    M, S = case["rows"], case["segments"]
    if case["op"] == "adapter":
        dr.dr_adapter(s["desc"], M, s["x"], s["x"].stride(0), s["w"], s["bias"], s["a"], s["b"], s["scale"], S, s["row_start"], s["adapter"],
                      s["y"], s["y"].stride(0), s["t"], None, s["ws"], s["ws"].numel())
        return s["y"] if s["t"] is None else (s["y"], s["t"])
    dr.dr_adapter_bwd(s["desc"], M, s["dy"], s["dy"].stride(0), s["x"], s["x"].stride(0), s["w"], s["a"], s["b"], s["scale"], S, s["row_start"],
                      s["adapter"], s["t"], s["dx"], s["dx"].stride(0), s["da"], s["db"], None, s["ws"], s["ws"].numel())
    return s["dx"], s["da"], s["db"]


def _kept(s, rows, channels):
    """The dropout's factors in float64, from the generator's definition in numpy's unsigned arithmetic."""
    p = s["case"]["p"]
    if not p:
        return None
    n = rows * channels
    e = np.arange((n + 7) // 8, dtype=np.uint64)
    low, c32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    x0, x1 = e & low, e >> c32
    x2, x3 = np.full_like(e, s["offset"] & 0xFFFFFFFF), np.full_like(e, s["offset"] >> 32)
    for r in range(10):
        key0 = np.uint64((s["seed"] + r * 0x9E3779B9) & 0xFFFFFFFF)
        key1 = np.uint64(((s["seed"] >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (b >> c32) ^ x1 ^ key0, b & low, (a >> c32) ^ x3 ^ key1, a & low
    words = np.stack([x0, x1, x2, x3], 1).astype("<u4").view("<u2").reshape(-1)[:n].reshape(rows, channels)
    keep = torch.from_numpy(words.astype(np.int32)).cuda() >= _threshold(p)
    return keep.double() / (1 - _threshold(p) / 65536)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        y = torch.mul(s["x"].double(), _kept(s, case["rows"], case["channels"]))
        return y if s["residual"] is None else y.add_(s["residual"].double())
    M, K = case["rows"], case["cin"]
    f = _kept(s, M, K)
    first, last = s["starts"][0], s["starts"][-1]
    x, w = s["x"].double(), s["w"].double()
    xd = x if f is None else x * f
    # each request on its own, in the order of its rows
    spans = [(u, v, a) for u, v, a in zip(s["starts"], s["starts"][1:], s["ids"]) if v > u and a >= 0]
    if case["op"] == "adapter":
        y, t = s["y"].double(), torch.zeros((M, case["rank"]), dtype=torch.float64, device="cuda")
        y[first:last] = torch.addmm(s["bias"].double(), x[first:last], w.mT)
        for u, v, a in spans:
            t[u:v] = torch.einsum("mk,rk->mr", xd[u:v], s["a"][a].double())
            y[u:v] += torch.einsum("mr,nr->mn", t[u:v] * s["scale"][a].double(), s["b"][a].double())
        if case["relu"]:
            y[first:last] = y[first:last].relu()
        return y if s["t"] is None else (y, t)
    dy, t = s["dy"].double(), s["t"].double()
    dx = s["dx"].double()
    dx[first:last] = dy[first:last] @ w
    da = torch.zeros(s["a"].shape, dtype=torch.float64, device="cuda")
    db = torch.zeros(s["b"].shape, dtype=torch.float64, device="cuda")
    for u, v, a in spans:
        sdy = dy[u:v] * s["scale"][a].double()
        up = torch.einsum("mn,nr->mr", sdy, s["b"][a].double())
        back = torch.einsum("mr,rk->mk", up, s["a"][a].double())
        dx[u:v] += back if f is None else back * f[u:v]
        da[a] += torch.einsum("mr,mk->rk", up, xd[u:v])
        db[a] += torch.einsum("mn,mr->nr", sdy, t[u:v])
    return dx, da, db
