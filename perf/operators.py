"""Cases of two serving operators for a batch whose tokens belong to different requests:

  layer    a whole MoE layer for a few tokens (layer_tokens): router, the selected experts'
           SwiGLU FFNs out of a slot pool, an always-active shared expert, the weighted sum
  adapter  a projection that all tokens share, with each token's own low-rank adapter
           beside it (adapter_project), from single tokens to long prompts

Formulas (t a token; all sums in 32 bits or more):
  layer    l = Wr x_t, S the k largest (ties to the lower id), g = softmax of l over S
           y_t = y_in_t + sum_{e in S} g_e FFN_e(x_t) + FFN_shared(x_t), where
           FFN(x) = W2 (SiLU(W1 x) * W3 x); an expert without a slot contributes nothing
  adapter  y_t = y_in_t + W x_t + scale_a B_a (A_a x_t), a = adapters[t] (none if negative)

Weights are bf16; x and y are fp32 or bf16 ("act"). Sizes are those of the workloads this
repository is built around (tiny, Mixtral-8x7B, Phi-3.5-MoE, the fine-grained layer with a
shared expert) and generic ones around them.
"""
import math

import torch

own = False

DEV = "cuda"

MIXTRAL = dict(d=4096, f=14336, n=8, k=2, f_shared=0)
PHI = dict(d=4096, f=6400, n=16, k=2, f_shared=0)
FINE = dict(d=3584, f=2560, n=64, k=8, f_shared=20480)


def listed():
    return [
        # The smallest call: one token through the tiny layer. Launches and latency.
        dict(name="layer-tiny-1", kind="layer", T=1, d=256, f=512, n=4, k=2, f_shared=0, act="f32", cached=4, add=False),
        # Batch-1 decode with every expert resident: a wide and a fine-grained layer.
        dict(name="layer-mixtral-1", kind="layer", T=1, act="f32", cached=8, add=False, **MIXTRAL),
        dict(name="layer-fine-1", kind="layer", T=1, act="bf16", cached=64, add=True, **FINE),
        # Four requests on a layer whose cache holds 13 of 16 experts (the others run on the host).
        dict(name="layer-phi-4", kind="layer", T=4, act="bf16", cached=13, add=True, **PHI),
        # Ragged widths, between the named layers, an odd batch.
        dict(name="layer-ragged-11", kind="layer", T=11, d=1048, f=1816, n=60, k=4, f_shared=2648, act="f32", cached=60,
             add=True),
        # A full batch on the fine-grained layer: some 42 of 64 experts are read.
        dict(name="layer-fine-8", kind="layer", T=8, act="f32", cached=64, add=False, **FINE),
        # One token through a small projection with an adapter: latency.
        dict(name="adapter-small-1", kind="adapter", T=1, d=256, o=512, r=8, n=4, act="f32", spread="each", add=False),
        # Decode batches beside an expert's up and down matrices, each token an adapter of its own.
        dict(name="adapter-up-8", kind="adapter", T=8, d=4096, o=14336, r=16, n=8, act="f32", spread="each", add=False),
        dict(name="adapter-down-16", kind="adapter", T=16, d=14336, o=4096, r=64, n=32, act="bf16", spread="each", add=True),
        # A mixed step: prompts of several requests and single tokens, ragged widths, fp32 states.
        dict(name="adapter-ragged-333", kind="adapter", T=333, d=3592, o=2568, r=24, n=9, act="f32", spread="runs", add=True),
        # Prompts of several requests: 512 tokens, and a long one (the largest case).
        dict(name="adapter-up-512", kind="adapter", T=512, d=4096, o=14336, r=32, n=8, act="bf16", spread="runs", add=False),
        dict(name="adapter-down-4096", kind="adapter", T=4096, d=14336, o=4096, r=64, n=16, act="bf16", spread="runs",
             add=True),
    ]


# ------------------------------------------------------------------ drawn cases
_MAX_POOL = 2.9e9       # bytes of a drawn layer's experts
_MAX_FLOPS = 4.8e11     # of a drawn projection (the long listed one)


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread evenly over its logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + step * 0.99)))
    return min(hi, max(lo, int(v // step) * step))


def draw(rng):
    act, add = rng.choice(["f32", "bf16"]), rng.random() < 0.5
    if rng.random() < 0.5:
        d = _log(rng, 256, 8192, 8)
        T = rng.randint(1, min(16, 32768 // d))
        n = rng.choice([4, 8, 12, 16, 32, 60, 64, 128, 200])
        k = rng.randint(1, min(8, n // 2))
        f = _log(rng, 256, 14336, 8)
        while n * 6.0 * d * f > _MAX_POOL:
            f = max(8, f // 2 // 8 * 8)
        fs = rng.choice([0, _log(rng, 256, 20480 if d < 4000 else 8192, 8)])
        cached = n if rng.random() < 0.6 else rng.randint(n // 2, n)
        return dict(kind="layer", T=T, d=d, f=f, n=n, k=k, f_shared=fs, act=act, cached=cached, add=add)
    d, o = _log(rng, 128, 14336, 8), _log(rng, 128, 14336, 8)
    T = rng.randint(1, 16) if rng.random() < 0.5 else _log(rng, 17, 4096)
    while 2.0 * T * d * o * (3 if act == "f32" else 1) > _MAX_FLOPS:
        T = max(1, T // 2)
    return dict(kind="adapter", T=T, d=d, o=o, r=rng.choice([8, 16, 24, 32, 64, 128]), n=rng.randint(1, 48), act=act,
                spread=rng.choice(["each", "runs"]), add=add)


# ------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["act"] == "f32" else torch.bfloat16


def _slab_values(d, f):
    """bf16 values of a slab W1 [f][d] | W3 [f][d] | W2 [d][f] with its padding to 256 bytes."""
    return (6 * d * f + 255) // 256 * 128


def _inputs(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, device=DEV, dtype=dtype).normal_(0.0, std, generator=g)

    T, d = c["T"], c["d"]
    s = dict(x=normal(T, d).to(_dtype(c)))
    if c["kind"] == "layer":
        n, f, fs = c["n"], c["f"], c["f_shared"]
        std = 0.02 if d >= 1024 else d ** -0.5
        s["wr"] = normal(n, d, std=d ** -0.5)
        # a cache smaller than the layer: `cached` slots hold the experts in a random order
        order = torch.empty(n, device=DEV).uniform_(generator=g).argsort()
        slotmap = torch.full((n,), -1, dtype=torch.int32, device=DEV)
        slotmap[order[:c["cached"]]] = torch.arange(c["cached"], dtype=torch.int32, device=DEV)
        s["slotmap"] = slotmap
        s["pool"] = normal(c["cached"], _slab_values(d, f), std=std, dtype=torch.bfloat16)
        s["shared"] = normal(_slab_values(d, fs), std=std, dtype=torch.bfloat16) if fs else None
        s["y_in"] = normal(T, d).to(_dtype(c)) if c["add"] else None
        return s
    n, r, o = c["n"], c["r"], c["o"]
    s["w"] = normal(o, d, std=d ** -0.5, dtype=torch.bfloat16)
    s["a"] = normal(n, r, d, std=d ** -0.5, dtype=torch.bfloat16)
    s["b"] = normal(n, o, r, std=0.5 * r ** -0.5, dtype=torch.bfloat16)
    s["scale"] = torch.empty(n, device=DEV).uniform_(0.5, 2.0, generator=g)
    # whose token: each its own draw, or prompts one after the other; -1 is the plain model
    if c["spread"] == "each":
        ids = torch.empty(T, device=DEV).uniform_(-0.5, n, generator=g).floor().to(torch.int32)
    else:
        runs = min(T, n + 1)
        cuts = torch.empty(runs - 1, device=DEV).uniform_(0, T, generator=g).floor()
        run = (torch.arange(T, device=DEV)[:, None] >= cuts[None, :]).sum(1)
        who = torch.empty(n + 1, device=DEV).uniform_(generator=g).argsort().to(torch.int32) - 1
        ids = who[run]
    s["ids"] = ids.contiguous()
    s["y_in"] = normal(T, o).to(_dtype(c)) if c["add"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = c = case
    T, d = c["T"], c["d"]
    if not own:
        return s
    import paper_2512_16473_amd as moe
    if c["kind"] == "layer":
        nbytes = moe.layer_tokens_workspace_bytes(T, d, c["f"], c["n"], c["k"], c["f_shared"])
        s["idx"] = torch.empty((T, c["k"]), dtype=torch.int32, device=DEV)
        s["g"] = torch.empty((T, c["k"]), device=DEV)
        s["y"] = torch.empty((T, d), dtype=_dtype(c), device=DEV)
    else:
        nbytes = moe.adapter_workspace_bytes(T, d, c["o"], c["r"], _dtype(c))
        s["y"] = torch.empty((T, c["o"]), dtype=_dtype(c), device=DEV)
    s["ws"] = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    c = s["case"]
    if own:
        import paper_2512_16473_amd as moe
        if c["kind"] == "layer":
            moe.layer_tokens(s["x"], s["wr"], s["pool"], c["f"], c["k"], s["y"], s["ws"], n_slots=c["cached"],
                             slotmap=s["slotmap"], shared=s["shared"], f_shared=c["f_shared"], y_in=s["y_in"],
                             idx=s["idx"], w=s["g"])
            return dict(y=s["y"], idx=s["idx"], w=s["g"])
        moe.adapter_project(s["x"], s["w"], s["a"], s["b"], s["ids"], s["y"], s["ws"], scale=s["scale"], y_in=s["y_in"])
        return dict(y=s["y"])
    return _plain_layer(s, c) if c["kind"] == "layer" else _plain_adapter(s, c)


def _matrices(pool, d, f):
    """W1 [n][f][d], W3 [n][f][d], W2 [n][d][f] of a pool of slabs [n][values]."""
    return (pool[:, :f * d].unflatten(1, (f, d)), pool[:, f * d:2 * f * d].unflatten(1, (f, d)),
            pool[:, 2 * f * d:3 * f * d].unflatten(1, (d, f)))


def _ffn(w1, w3, w2, x):
    """x [m][d] through one expert's matrices, in fp32."""
    a, b = x @ w1.float().t(), x @ w3.float().t()
    return (a / (1.0 + torch.exp(-a)) * b) @ w2.float().t()


def _plain_layer(s, c):
    T, d, f, fs, k = c["T"], c["d"], c["f"], c["f_shared"], c["k"]
    x = s["x"].float()
    # 64 bits: experts next to the border of the top k keep their order
    l = x.double() @ s["wr"].double().t()
    top, idx = torch.sort(l, dim=1, descending=True, stable=True)
    top, idx = top[:, :k], idx[:, :k]
    g = torch.exp(top - top[:, :1])
    g = (g / g.sum(1, keepdim=True)).float()
    slots = s["slotmap"].long()[idx]
    y = s["y_in"].float() if c["add"] else torch.zeros((T, d), device=DEV)
    y = y.clone()
    w1, w3, w2 = _matrices(s["pool"], d, f)
    for t in range(T):
        for j in range(k):
            at = slots[t, j:j + 1]
            e = at.clamp(min=0)
            v = _ffn(w1.index_select(0, e)[0], w3.index_select(0, e)[0], w2.index_select(0, e)[0], x[t:t + 1])[0]
            y[t] += torch.where(at >= 0, g[t, j] * v, 0.0 * v)
    if fs:
        w1, w3, w2 = _matrices(s["shared"][None], d, fs)
        y += _ffn(w1[0], w3[0], w2[0], x)
    return dict(y=y.to(s["x"].dtype), idx=idx.to(torch.int32), w=g)


def _plain_adapter(s, c):
    x = s["x"].float()
    y = x @ s["w"].float().t()
    ids = s["ids"]
    for a in range(c["n"]):
        v = (x @ s["a"][a].float().t()) * s["scale"][a]
        y = torch.where((ids == a)[:, None], y + v @ s["b"][a].float().t(), y)
    if c["add"]:
        y = y + s["y_in"].float()
    return dict(y=y.to(s["x"].dtype))


# ------------------------------------------------------------------ floors
def work(case):
    """Each input read once (of the experts and adapters those that a batch of unrelated
    tokens selects on average), each output written once."""
    c = case
    T, d, act = c["T"], c["d"], 4 if c["act"] == "f32" else 2
    if c["kind"] == "layer":
        n, k, f, fs = c["n"], c["k"], c["f"], c["f_shared"]
        here = c["cached"] / n
        read = n * (1.0 - (1.0 - k / n) ** T) * here
        nbytes = 6.0 * d * (f * read + fs) + 4.0 * n * d + T * d * act * (3 if c["add"] else 2) + 8.0 * T * k + 4.0 * n
        return {"bytes": nbytes, "flops": T * (6.0 * d * (f * k * here + fs) + 2.0 * n * d)}
    o, r, n = c["o"], c["r"], c["n"]
    used = n * (1.0 - (1.0 - 1.0 / (n + 0.5)) ** T) if c["spread"] == "each" else min(T, n + 1) * n / (n + 1.0)
    share = n / (n + 0.5) if c["spread"] == "each" else n / (n + 1.0)
    nbytes = 2.0 * d * o + used * (2.0 * r * (d + o) + 4) + T * act * (d + o * (2 if c["add"] else 1)) + 4.0 * T
    return {"bytes": nbytes, "flops": 2.0 * T * (d * o + share * r * (d + o))}


# ------------------------------------------------------------------ the results in 64 bits
def exact(case, seed):
    c = case
    s = _inputs(case, seed)
    x = s["x"].double()
    T, d = c["T"], c["d"]
    y = s["y_in"].double().clone() if c["add"] else None
    if c["kind"] == "adapter":
        out = torch.zeros((T, c["o"]), dtype=torch.float64, device=DEV) if y is None else y
        for lo in range(0, c["o"], 2048):
            out[:, lo:lo + 2048] += torch.mm(x, s["w"][lo:lo + 2048].double().t())
        ids = s["ids"].long()
        for a in sorted(set(ids.tolist()) - {-1}):
            mine = (ids == a).nonzero()[:, 0]
            low = torch.mm(x[mine], s["a"][a].double().t())
            out[mine] += float(s["scale"][a]) * torch.mm(low, s["b"][a].double().t())
        return dict(y=out)
    f, fs, k = c["f"], c["f_shared"], c["k"]
    out = torch.zeros((T, d), dtype=torch.float64, device=DEV) if y is None else y
    logits = (x[:, None, :] * s["wr"].double()[None]).sum(-1).cpu().tolist()
    where = s["slotmap"].tolist()
    chosen, gates = [], []
    for row in logits:
        best = sorted(range(c["n"]), key=lambda e: (-row[e], e))[:k]
        p = [math.exp(row[e] - row[best[0]]) for e in best]
        chosen.append(best)
        gates.append([v / sum(p) for v in p])

    def ffn(slab, width, rows):
        m = slab[:3 * d * width].view(3, -1)
        a = torch.mm(rows, m[0].view(width, d).double().t())
        b = torch.mm(rows, m[1].view(width, d).double().t())
        return torch.mm(a * torch.sigmoid(a) * b, m[2].view(d, width).double().t())

    for e in range(c["n"]):
        users = [(t, chosen[t].index(e)) for t in range(T) if e in chosen[t]]
        if not users or where[e] < 0:
            continue
        ts = torch.tensor([t for t, _ in users], device=DEV)
        gs = torch.tensor([gates[t][j] for t, j in users], dtype=torch.float64, device=DEV)
        out[ts] += gs[:, None] * ffn(s["pool"][where[e]], f, x[ts])
    if fs:
        out += ffn(s["shared"], fs, x)
    return dict(y=out, idx=torch.tensor(chosen, dtype=torch.int32, device=DEV),
                w=torch.tensor(gates, dtype=torch.float64, device=DEV))
