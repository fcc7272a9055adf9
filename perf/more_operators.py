"""The operators that make the features the lookup pairs, and their gradients: what a flow network's program calls between its convolutions
and the pyramid's build, from one token to an 8K frame's map.

A case is one of
    group_norm           y = act(norm over a group's channels and all pixels of x, times weight, plus bias); with "train" also the statistics
    group_norm_backward  its gradients with respect to x, weight and bias
    gated                y = act(x wg^T + bg) * (x wu^T + bu); with "train" also both sums, which the gradient reads
    gated_backward       its gradients with respect to x, w and bias
    attention            softmax(scale q k^T) v per head over the keys of another map or encoder, whose number, lengths and mask are its
                         own; with "train" also the logarithm of each row's sum, which the gradient reads
    attention_backward   its gradients with respect to q, k and v
Rows are the pixels of channels-last maps, or tokens.  Vectors and statistics are fp32 in every case, as the library takes them.
"""
import math

import torch

#: set from outside: whether run() calls the library or computes the plain forms
own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid")
EPS = 1e-5
#: the most that a drawn case multiplies and holds, below the largest listed one
MOST_PRODUCTS = 200 * 10 ** 9
MOST_ELEMENTS = 1 << 27


def listed():
    return [
        # one pair's small crop behind the encoder's first block: launches and latency
        {"name": "group-norm-46x62-f16", "kind": "group_norm", "type": "f16", "B": 2, "P": 46 * 62, "C": 64, "G": 8, "act": "relu"},
        # an 8K frame's features, the pair as one batch, in training: the statistics are kept
        {"name": "group-norm-2x540x960-bf16", "kind": "group_norm", "type": "bf16", "B": 2, "P": 540 * 960, "C": 256, "G": 32, "act": "relu",
         "train": True},
        # odd maps, groups of three channels, fp32
        {"name": "group-norm-4x47x155-f32-grad", "kind": "group_norm_backward", "type": "f32", "B": 4, "P": 47 * 155, "C": 96, "G": 32,
         "act": "silu"},
        # a pair at 4K in training
        {"name": "group-norm-2x270x480-bf16-grad", "kind": "group_norm_backward", "type": "bf16", "B": 2, "P": 270 * 480, "C": 128, "G": 8,
         "act": "relu"},
        # one token: every weight is read for one row
        {"name": "gated-token-1024x4096-bf16", "kind": "gated", "type": "bf16", "M": 1, "K": 1024, "N": 4096, "act": "silu"},
        # the feed-forward block's widening products at 1080p, in training
        {"name": "gated-135x240-bf16-train", "kind": "gated", "type": "bf16", "M": 32400, "K": 256, "N": 1024, "act": "silu", "train": True},
        # an odd number of rows in fp32
        {"name": "gated-2x47x155-f32", "kind": "gated", "type": "f32", "M": 14570, "K": 256, "N": 682, "act": "gelu"},
        # a 4K map's rows in training
        {"name": "gated-270x480-bf16-grad", "kind": "gated_backward", "type": "bf16", "M": 129600, "K": 256, "N": 512, "act": "gelu"},
        # one query of each of eight sequences on the encoder's states that are kept for it, eight heads on two, ragged lengths
        {"name": "attention-8x1x32768-bf16", "kind": "attention", "type": "bf16", "B": 8, "Lq": 1, "Lk": 32768, "H": 8, "HK": 2, "D": 128,
         "lengths": True},
        # every pixel of a 1080p map on every pixel of the other: the largest product
        {"name": "attention-135x240-bf16-train", "kind": "attention", "type": "bf16", "B": 1, "Lq": 32400, "Lk": 32400, "H": 2, "HK": 2,
         "D": 128, "train": True},
        # small crops whose right and lower borders are padding, against a map of another size, fp32, in training
        {"name": "attention-2x46x62-47x155-f32-grad", "kind": "attention_backward", "type": "f32", "B": 2, "Lq": 46 * 62, "Lk": 47 * 155,
         "H": 4, "HK": 4, "D": 64, "mask": 155},
        # a 720p pair in training
        {"name": "attention-2x90x160-bf16-grad", "kind": "attention_backward", "type": "bf16", "B": 2, "Lq": 14400, "Lk": 14400, "H": 2,
         "HK": 2, "D": 64},
    ]


def _log_int(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm; two of three are multiples of eight where there is room."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))
    v = max(lo, min(hi, int(v)))
    return max(8, v & ~7) if v >= 64 and rng.random() < 2 / 3 else v


def draw(rng):
    kind = rng.choice(("group_norm", "group_norm_backward", "gated", "gated_backward", "attention", "attention", "attention_backward"))
    typ = rng.choice(("f32", "bf16", "bf16", "f16"))
    slow = (4 if typ == "f32" else 1) * (3 if kind.endswith("backward") else 1)
    if kind.startswith("group_norm"):
        width = rng.choice((1, 2, 3, 4, 6, 8, 8, 16, 16, 32, 64))
        G = _log_int(rng, 1, 512 // width)
        B = _log_int(rng, 1, 16)
        case = {"kind": kind, "type": typ, "B": B, "P": _log_int(rng, 16, min(540 * 960, MOST_ELEMENTS // (B * G * width))), "C": G * width,
                "G": G, "act": rng.choice(ACTS)}
        if kind == "group_norm":
            case["train"] = rng.random() < 0.5
        return case
    if kind.startswith("gated"):
        N, K = _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)
        most = min(540 * 960, MOST_ELEMENTS // max(2 * N, K), MOST_PRODUCTS // (slow * 2 * N * K))
        case = {"kind": kind, "type": typ, "M": _log_int(rng, 1, most), "K": K, "N": N, "act": rng.choice(ACTS)}
        if kind == "gated":
            case["train"] = rng.random() < 0.4
        case["bias"] = rng.random() < 0.6
        return case
    D = rng.choice((32, 64, 64, 128, 128, 256, 40, 72, 96, 160))
    HK = rng.choice((1, 1, 2, 4, 8))
    H = HK * rng.choice((1, 1, 1, 2, 3, 4))
    B = rng.choice((1, 1, 2, 3, 8))
    Lk = _log_int(rng, 1, min(32768, MOST_ELEMENTS // (B * HK * D)))
    most = min(32400, MOST_PRODUCTS // (slow * 2 * B * H * D * Lk), MOST_ELEMENTS // (B * H * D))
    case = {"kind": kind, "type": typ, "B": B, "Lq": _log_int(rng, 1, most), "Lk": Lk, "H": H, "HK": HK, "D": D,
            "lengths": rng.random() < 0.4}
    if rng.random() < 0.4:
        case["mask"] = _log_int(rng, 1, Lk)
    if kind == "attention":
        case["train"] = rng.random() < 0.4
    return case


def _lengths(case):
    """How many keys each item has: from all of them down to a few, and none for the last of three and more."""
    B, Lk = case["B"], case["Lk"]
    if not case.get("lengths"):
        return [Lk] * B
    return [0 if b >= 2 and b == B - 1 else max(1, Lk - b * Lk // (B + 1)) for b in range(B)]


def _mask(case, b):
    """Item b's keys as rows of a map `mask` pixels wide, of which an eighth (a quarter, ...) of rows and columns is padding."""
    width, Lk = case["mask"], case["Lk"]
    keep = 8 - (b + 1) % 4
    rows = -(-Lk // width)
    i = torch.arange(Lk)
    return (i // width * 8 < rows * keep) & (i % width * 8 < width * keep)


def _counts(case):
    """Keys that count, per item."""
    if "mask" not in case:
        return _lengths(case)
    return [int(_mask(case, b)[:n].sum()) for b, n in enumerate(_lengths(case))]


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    T = DTYPES[case["type"]]

    def normal(shape, sigma=1.0, dtype=T, mean=0.0):
        return torch.randn(shape, device=dev, generator=g, dtype=torch.float32).mul_(sigma).add_(mean).to(dtype)

    st = dict(case)
    kind = case["kind"]
    if kind.startswith("group_norm"):
        B, P, C = case["B"], case["P"], case["C"]
        # a convolution's output: channels with means and spreads of their own
        st["x"] = (normal((B, P, C), 1.0, torch.float32) * (0.5 + torch.rand((C,), device=dev, generator=g))
                   + normal((C,), 1.0, torch.float32)).to(T)
        st["w"], st["b"] = normal((C,), 0.1, torch.float32, 1.0), normal((C,), 0.1, torch.float32)
        if kind == "group_norm_backward":
            st["dy"] = normal((B, P, C), 0.05)
            st["stats"] = _group_stats64(st["x"], case["G"]).float()
        return st
    if kind.startswith("gated"):
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = normal((M, K))
        st["w"] = normal((2 * N, K), K ** -0.5)
        st["b"] = normal((2 * N,), 0.1, torch.float32) if case.get("bias", True) else None
        if kind == "gated_backward":
            # sums of many terms: normal; what the forward pass left
            st["z"] = normal((M, 2 * N))
            st["dy"] = normal((M, N), 0.05)
        return st
    B, Lq, Lk, H, HK, D = (case[n] for n in ("B", "Lq", "Lk", "H", "HK", "D"))
    # scores of a spread of two, so that some keys count and most hardly do
    st["q"], st["k"], st["v"] = normal((B, Lq, H, D), 2.0), normal((B, Lk, HK, D)), normal((B, Lk, HK, D))
    st["scale"] = D ** -0.5
    st["k_lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=dev) if case.get("lengths") else None
    st["key_mask"] = torch.stack([_mask(case, b) for b in range(B)]).to(device=dev, dtype=torch.uint8) if "mask" in case else None
    if kind == "attention_backward":
        st["do"] = normal((B, Lq, H, D), 0.05)
        st["o"], st["lse"] = _attention_plain(dict(st, kind="attention", train=True))
    return st


# ---------------------------------------------------------------- the library's calls

def _own(st):
    from paper_2505_16942_amd import binding as cb
    kind = st["kind"]
    if kind.startswith("attention"):
        kw = dict(scale=st["scale"], k_lengths=st["k_lengths"], key_mask=st["key_mask"])
        if kind == "attention_backward":
            return list(cb.corr_attention_backward(st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"], **kw))
        if st.get("train"):
            lse = torch.empty((st["B"], st["H"], st["Lq"]), dtype=torch.float32, device=st["q"].device)
            return [cb.corr_attention(st["q"], st["k"], st["v"], lse=lse, **kw), lse]
        return [cb.corr_attention(st["q"], st["k"], st["v"], **kw)]
    act = getattr(cb, "CORR_ACT_" + st["act"].upper())
    if kind == "group_norm":
        if st.get("train"):
            stats = torch.empty((st["B"], st["G"], 2), dtype=torch.float32, device=st["x"].device)
            return [cb.corr_group_norm(st["x"], st["G"], weight=st["w"], bias=st["b"], act=act, eps=EPS, stats=stats), stats]
        return [cb.corr_group_norm(st["x"], st["G"], weight=st["w"], bias=st["b"], act=act, eps=EPS)]
    if kind == "group_norm_backward":
        return list(cb.corr_group_norm_backward(st["x"], st["G"], st["stats"], st["dy"], weight=st["w"], bias=st["b"], act=act))
    if kind == "gated":
        if st.get("train"):
            z = torch.empty((st["M"], 2 * st["N"]), dtype=st["x"].dtype, device=st["x"].device)
            return [cb.corr_gated_linear(st["x"], st["w"], bias=st["b"], act=act, preact=z), z]
        return [cb.corr_gated_linear(st["x"], st["w"], bias=st["b"], act=act)]
    got = cb.corr_gated_linear_backward(st["x"], st["w"], st["dy"], st["z"], act=act, want_bias=st["b"] is not None)
    return [t for t in got if t is not None]


# ---------------------------------------------------------------- plain forms: fp32 (long sums fp64), rounded once

def _act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    return z


def _act_grad(z, name):
    """Derivative of _act; None stands for one everywhere."""
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "sigmoid":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 - s)
    return None


def _by_group(v, G):
    """[B, P, C] as [B, P, G, C / G]"""
    return v.reshape(v.shape[0], v.shape[1], G, v.shape[2] // G)


def _group_plain(st):
    T, B, P, C, G = st["x"].dtype, st["B"], st["P"], st["C"], st["G"]
    x = _by_group(st["x"].float(), G)
    w, b = st["w"].view(G, C // G), st["b"].view(G, C // G)
    if st["kind"] == "group_norm":
        mean = x.mean((1, 3), keepdim=True, dtype=torch.float64).float()
        x = x - mean
        rho = (x.square().mean((1, 3), keepdim=True, dtype=torch.float64).float() + EPS).rsqrt()
        y = _act(x * rho * w + b, st["act"]).reshape(B, P, C).to(T)
        return [y, torch.cat([mean, rho], 3).view(B, G, 2)] if st.get("train") else [y]
    mean, rho = st["stats"][:, None, :, :1], st["stats"][:, None, :, 1:]
    hat = (x - mean) * rho
    dz = _by_group(st["dy"].float(), G)
    slope = _act_grad(hat * w + b, st["act"])
    if slope is not None:
        dz = dz * slope
    long = lambda v, dims, keep: v.sum(dims, keepdim=keep, dtype=torch.float64).float()  # noqa: E731
    q = dz * w
    n = P * (C // G)
    dx = rho * (q - long(q, (1, 3), True) / n - hat * (long(q * hat, (1, 3), True) / n))
    return [dx.reshape(B, P, C).to(T), long(dz * hat, (0, 1), False).reshape(C), long(dz, (0, 1), False).reshape(C)]


def _gated_plain(st):
    T, N = st["x"].dtype, st["N"]
    x, w = st["x"].float(), st["w"].float()
    if st["kind"] == "gated":
        z = x @ w.t()
        if st["b"] is not None:
            z = z + st["b"]
        y = (_act(z[:, :N], st["act"]) * z[:, N:]).to(T)
        return [y, z.to(T)] if st.get("train") else [y]
    z, dy = st["z"].float(), st["dy"].float()
    up = dy * z[:, N:]
    slope = _act_grad(z[:, :N], st["act"])
    dz = torch.cat([up if slope is None else up * slope, dy * _act(z[:, :N], st["act"])], 1)
    out = [(dz @ w).to(T), (dz.t() @ x).to(T)]
    if st["b"] is not None:
        out.append(dz.sum(0, dtype=torch.float64).float())
    return out


def _valid(st, b):
    """The keys of item b that count, [Lk] of truth values, or None for all."""
    keep = None
    if st["k_lengths"] is not None:
        keep = torch.arange(st["Lk"], device=st["q"].device) < st["k_lengths"][b]
    if st["key_mask"] is not None:
        m = st["key_mask"][b] != 0
        keep = m if keep is None else keep & m
    return keep


#: scores that the plain form holds at a time
PLAIN_SCORES = 1 << 29


def _attention_plain(st):
    T, (B, Lq, H, D), Lk = st["q"].dtype, st["q"].shape, st["Lk"]
    per = H // st["HK"]
    back = st["kind"] == "attention_backward"
    step = max(1, PLAIN_SCORES // Lk)
    if back:
        dq, dk, dv = (torch.zeros(t.shape, dtype=torch.float32, device=t.device) for t in (st["q"], st["k"], st["v"]))
    else:
        out = torch.empty((B, Lq, H, D), dtype=torch.float32, device=st["q"].device)
        lse = torch.empty((B, H, Lq), dtype=torch.float32, device=st["q"].device)
    for b in range(B):
        keep = _valid(st, b)
        for h in range(H):
            k, v = st["k"][b, :, h // per].float(), st["v"][b, :, h // per].float()
            for lo in range(0, Lq, step):
                rows = slice(lo, min(Lq, lo + step))
                q = st["q"][b, rows, h].float()
                s = (q @ k.t()).mul_(st["scale"])
                if back:
                    low = st["lse"][b, h, rows, None]
                    p = torch.exp(s - torch.where(low == -math.inf, 0.0, low))
                    if keep is not None:
                        p = torch.where(keep, p, 0.0)
                    do = st["do"][b, rows, h].float()
                    dv[b, :, h // per] += p.t() @ do
                    delta = (do * st["o"][b, rows, h].float()).sum(1, keepdim=True)
                    ds = p.mul_((do @ v.t()).sub_(delta))
                    dq[b, rows, h] = (ds @ k).mul_(st["scale"])
                    dk[b, :, h // per] += (ds.t() @ q).mul_(st["scale"])
                    continue
                if keep is not None:
                    s = torch.where(keep, s, -math.inf)
                top = s.max(1, keepdim=True).values
                top = torch.where(top == -math.inf, 0.0, top)
                p = s.sub_(top).exp_()
                total = p.sum(1, keepdim=True)
                out[b, rows, h] = (p @ v) / torch.where(total == 0, 1.0, total)
                lse[b, h, rows] = (total.log() + top)[:, 0]
    if back:
        return [dq.to(T), dk.to(T), dv.to(T)]
    return [out.to(T), lse] if st.get("train") else [out.to(T)]


def run(state):
    if own:
        return _own(state)
    if state["kind"].startswith("group_norm"):
        return _group_plain(state)
    return _gated_plain(state) if state["kind"].startswith("gated") else _attention_plain(state)


def work(case):
    e, kind = {"f32": 4, "bf16": 2, "f16": 2}[case["type"]], case["kind"]
    if kind.startswith("group_norm"):
        elements, small = case["B"] * case["P"] * case["C"], 8 * case["C"]
        stats = 8 * case["B"] * case["G"]
        if kind == "group_norm":
            return {"bytes": 2 * e * elements + small + (stats if case.get("train") else 0), "flops": 10 * elements}
        return {"bytes": 3 * e * elements + 2 * small + stats, "flops": 20 * elements}
    if kind.startswith("gated"):
        M, N, K = case["M"], case["N"], case["K"]
        bias = 8 * N if case.get("bias", True) else 0
        if kind == "gated":
            return {"bytes": e * (M * K + 2 * N * K + M * N * (3 if case.get("train") else 1)) + bias, "flops": 4 * M * N * K}
        return {"bytes": e * (2 * M * K + 4 * N * K + 3 * M * N) + bias, "flops": 8 * M * N * K}
    B, Lq, H, HK, D = (case[n] for n in ("B", "Lq", "H", "HK", "D"))
    keys = sum(_counts(case))
    rows, small = B * Lq * H, (B * case["Lk"] if "mask" in case else 0) + (4 * B if case.get("lengths") else 0)
    if kind == "attention":
        return {"bytes": e * D * (2 * rows + 2 * keys * HK) + small + (4 * rows if case.get("train") else 0), "flops": 4 * Lq * H * keys * D}
    # gradients of keys that do not count are written too
    return {"bytes": e * D * (4 * rows + 2 * keys * HK + 2 * B * case["Lk"] * HK) + 4 * rows + small, "flops": 10 * Lq * H * keys * D}


# ---------------------------------------------------------------- the definition in 64 bits

def _phi(z):
    return torch.special.ndtr(z)


def _twice(z):
    return math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)


#: name: (value, derivative), of float64 tensors
_EXACT_ACTS = {
    "none": (lambda z: z, torch.ones_like),
    "relu": (torch.relu, lambda z: torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))),
    "gelu": (lambda z: z * _phi(z), lambda z: _phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)),
    # 0.5 (1 + tanh u) = sigmoid(2 u)
    "gelu_tanh": (lambda z: z * torch.sigmoid(_twice(z)),
                  lambda z: torch.sigmoid(_twice(z)) * (1 + z * torch.sigmoid(-_twice(z)) * math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2))),
    "silu": (lambda z: z * torch.sigmoid(z), lambda z: torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))),
    "sigmoid": (torch.sigmoid, lambda z: torch.sigmoid(z) * torch.sigmoid(-z)),
}


def _group_stats64(x, G):
    """[B, G, 2]: mean and 1 / spread, item by item"""
    out = []
    for item in x:
        v = item.double().view(item.shape[0], G, -1)
        n = v.shape[0] * v.shape[2]
        mu = v.sum((0, 2)) / n
        var = ((v - mu[:, None]) ** 2).sum((0, 2)) / n
        out.append(torch.stack([mu, 1 / torch.sqrt(var + EPS)], 1))
    return torch.stack(out)


def _group_exact(st):
    G, C, P = st["G"], st["C"], st["P"]
    f, fd = _EXACT_ACTS[st["act"]]
    w, b = st["w"].double().view(G, -1), st["b"].double().view(G, -1)
    back = st["kind"] == "group_norm_backward"
    stats = st["stats"].double() if back else _group_stats64(st["x"], G)
    items, dw, db = [], 0, 0
    for i in range(st["B"]):
        rho = stats[i, :, 1, None]
        unit = (st["x"][i].double().view(P, G, -1) - stats[i, :, 0, None]) * rho
        z = unit * w + b
        if not back:
            items.append(f(z).view(P, C))
            continue
        dz = st["dy"][i].double().view(P, G, -1) * fd(z)
        db, dw = db + dz.sum(0), dw + (dz * unit).sum(0)
        dunit = dz * w
        n = P * (C // G)
        inner = (dunit * unit).sum((0, 2)) / n
        dunit = dunit - (dunit.sum((0, 2)) / n)[:, None] - unit * inner[:, None]
        items.append((dunit * rho).view(P, C))
    if back:
        return [torch.stack(items), dw.view(C), db.view(C)]
    return [torch.stack(items), stats] if st.get("train") else [torch.stack(items)]


def _gated_exact(st):
    M, N, K = st["M"], st["N"], st["K"]
    wg, wu = st["w"][:N].double(), st["w"][N:].double()
    f, fd = _EXACT_ACTS[st["act"]]
    step = max(1, (1 << 25) // max(2 * N, K))
    rows, sums = [], None
    for lo in range(0, M, step):
        x = st["x"][lo:lo + step].double()
        if st["kind"] == "gated":
            gate, up = torch.mm(x, wg.t()), torch.mm(x, wu.t())
            if st["b"] is not None:
                gate, up = gate + st["b"][:N].double(), up + st["b"][N:].double()
            rows.append([f(gate) * up] + ([torch.cat([gate, up], 1)] if st.get("train") else []))
            continue
        z, dy = st["z"][lo:lo + step].double(), st["dy"][lo:lo + step].double()
        dgate, dup = dy * z[:, N:] * fd(z[:, :N]), dy * f(z[:, :N])
        rows.append([torch.mm(dgate, wg) + torch.mm(dup, wu)])
        both = torch.cat([dgate, dup], 1)
        part = [torch.mm(both.t().contiguous(), x)] + ([both.sum(0)] if st["b"] is not None else [])
        sums = part if sums is None else [p + q for p, q in zip(sums, part)]
    return [torch.cat(t) for t in zip(*rows)] + (sums or [])


def _attention_exact(st):
    B, Lq, H, D = st["q"].shape
    Lk, per = st["Lk"], H // st["HK"]
    back = st["kind"] == "attention_backward"
    dev = st["q"].device
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=dev)  # noqa: E731
    out, lse = new(B, Lq, H, D), torch.full((B, H, Lq), -math.inf, dtype=torch.float64, device=dev)
    dq, dk, dv = (new(*t.shape) if back else None for t in (st["q"], st["k"], st["v"]))
    step = max(1, (1 << 27) // Lk)
    for b in range(B):
        keep = _valid(st, b)
        at = torch.arange(Lk, device=dev) if keep is None else keep.nonzero()[:, 0]     # only the keys that count
        if not len(at):
            continue
        for h in range(H):
            k, v = st["k"][b, at, h // per].double(), st["v"][b, at, h // per].double()
            for lo in range(0, Lq, step):
                q = st["q"][b, lo:lo + step, h].double()
                s = torch.mm(q, k.t()) * st["scale"]
                total = torch.logsumexp(s, 1)
                p = torch.exp(s - total[:, None])
                o = torch.mm(p, v)
                if not back:
                    out[b, lo:lo + step, h], lse[b, h, lo:lo + step] = o, total
                    continue
                do = st["do"][b, lo:lo + step, h].double()
                dp = torch.mm(do, v.t())
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * st["scale"]
                dq[b, lo:lo + step, h] = torch.mm(ds, k)
                dk[b, :, h // per].index_add_(0, at, torch.mm(ds.t().contiguous(), q))
                dv[b, :, h // per].index_add_(0, at, torch.mm(p.t().contiguous(), do))
    if back:
        return [dq, dk, dv]
    return [out, lse] if st.get("train") else [out]


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("group_norm"):
        return _group_exact(st)
    return _gated_exact(st) if case["kind"].startswith("gated") else _attention_exact(st)
