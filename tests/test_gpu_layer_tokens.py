"""GPU tests of moe_layer_tokens (a whole MoE layer for a few tokens, routed on the device)
against its definition in 64 bits: routing, the selected experts' SwiGLU FFNs out of a slot
pool, the shared expert, and the sum.

Tolerance, per token. Products are exact (bf16 weights, fp32 activations in three bf16 parts)
and sums fp32, so a sum of K terms of random sign is off by about sqrt(K) roundings of its
size, 2^-24 each; the hidden values take two such sums (K = d), the output one (K = the
selected hidden columns). With a factor 8 for the largest of some thousand outputs:
8 * 2^-24 * (2 sqrt(d) + sqrt(columns)) of the output's RMS. A bf16 layer keeps hidden values
to 2^-17 (two parts, the second rounded: 2^-8 of 2^-8, halved), and rounds y once, by at most
2^-8 of its value."""
import numpy as np
import pytest

from _gpu_util import capture, say, side_streams, torch_cuda

pytestmark = pytest.mark.gpu

import paper_2512_16473_amd as moe  # noqa: E402


class Layer:
    """Seeded weights of a layer on the device: router, slot pool, slotmap, shared expert."""

    def __init__(self, torch, seed, d, f, n, k, fs=0, slots=None, wr=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.torch, self.d, self.f, self.n, self.k, self.fs = torch, d, f, n, k, fs
        def normal(std, *shape):
            return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)
        self.slots = list(range(n)) if slots is None else slots
        self.nslots = max(0, max(self.slots) + 1) if slots is not None else n
        self.slotmap = None if slots is None else torch.tensor(slots, dtype=torch.int32, device="cuda")
        self.wr = normal(d ** -0.5, n, d) if wr is None else wr.cuda()
        self.pool = normal(d ** -0.5, max(1, self.nslots), moe.slab_bytes(d, f) // 2).bfloat16()
        self.shared = normal(d ** -0.5, moe.slab_bytes(d, fs) // 2).bfloat16() if fs else None

    def ffn(self, slab, f, x):
        """[m][d] double -> [m][d] double"""
        d, s = self.d, slab.double()
        w1, w3, w2 = s[:f * d].view(f, d), s[f * d:2 * f * d].view(f, d), s[2 * f * d:3 * f * d].view(d, f)
        a = x @ w1.t()
        return (a * self.torch.sigmoid(a) * (x @ w3.t())) @ w2.t()

    def expect(self, x, y_in=None):
        """(y double [T][d], idx, w double, columns of each token)"""
        torch, T = self.torch, x.shape[0]
        xd = x.double()
        l = (xd[:, None, :] * self.wr.double()[None]).sum(-1).cpu().numpy()
        l = np.where(np.isnan(l), -np.inf, l)
        idx = np.stack([np.lexsort((np.arange(self.n), -row))[:self.k] for row in l])
        w = np.stack([np.exp(row[i] - row[i[0]]) for row, i in zip(l, idx)])
        w /= w.sum(1, keepdims=True)
        y = torch.zeros((T, self.d), dtype=torch.float64, device="cuda") if y_in is None else y_in.double().clone()
        cols = np.full(T, self.fs)
        for t in range(T):
            for e, g in zip(idx[t], w[t]):
                s = self.slots[e]
                if 0 <= s < self.nslots:
                    y[t] += g * self.ffn(self.pool[s], self.f, xd[t:t + 1])[0]
                    cols[t] += self.f
        if self.fs:
            y += self.ffn(self.shared, self.fs, xd)
        return y.cpu().numpy(), idx, w, cols

    def call(self, x, y, ws, y_in=None, idx=None, w=None, stream=None):
        return moe.layer_tokens(x, self.wr, self.pool, self.f, self.k, y, ws, n_slots=self.nslots, slotmap=self.slotmap,
                                shared=self.shared, f_shared=self.fs, y_in=y_in, idx=idx, w=w, stream=stream)

    def workspace(self, T):
        nbytes = moe.layer_tokens_workspace_bytes(T, self.d, self.f, self.n, self.k, self.fs)
        return self.torch.full((nbytes,), 0xFF, dtype=self.torch.uint8, device="cuda")   # any content

    def run(self, x, y_in=None):
        torch, T = self.torch, x.shape[0]
        y = torch.full((T, self.d), float("nan"), dtype=x.dtype, device="cuda")
        idx = torch.full((T, self.k), -7, dtype=torch.int32, device="cuda")
        w = torch.full((T, self.k), float("nan"), device="cuda")
        self.call(x, y, self.workspace(T), y_in, idx, w)
        torch.cuda.synchronize()
        return y, idx.cpu().numpy(), w.cpu().numpy()


def states(torch, seed, T, d, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty((T, d), device="cuda").normal_(generator=g).to(dtype)


def check(layer, x, y_in=None, what=""):
    y, idx, w = layer.run(x, y_in)
    ey, eidx, ew, cols = layer.expect(x, y_in)
    assert np.array_equal(idx, eidx), what
    assert np.all(np.abs(w - ew) <= 2.0 ** -23 * ew), what      # fp64 softmax rounded to fp32
    close(layer, y, ey, cols, what)
    return y


def close(layer, y, ey, cols, what):
    got = y.double().cpu().numpy()
    bf16 = y.dtype == layer.torch.bfloat16
    for t in range(got.shape[0]):
        rms = float(np.sqrt(np.mean(ey[t] ** 2)))
        tol = 8 * 2.0 ** -24 * (2 * layer.d ** 0.5 + float(cols[t]) ** 0.5) * rms
        if bf16:
            tol = tol + 2.0 ** -17 * 8 * rms + 2.0 ** -8 * np.abs(ey[t])
        err = np.abs(got[t] - ey[t])
        assert np.all(err <= tol), f"{what} t={t}: {float(np.max(err / np.maximum(tol, 1e-300))):.2f} x the tolerance"


SHAPES = [
    # d, f, n, k, fs, T
    (256, 512, 4, 2, 0, 1),          # the tiny layer
    (8, 8, 1, 1, 0, 1),              # one chunk, one short row block
    (264, 520, 5, 2, 0, 3),          # rows and columns that end inside a chunk; short row blocks
    (72, 136, 6, 3, 24, 16),         # most tokens; fewer chunks than waves; a tiny shared expert
    (1048, 1816, 12, 4, 264, 11),    # three column blocks of fp32
    (2048, 264, 32, 8, 0, 16),       # the T * d limit with 16 tokens
    (2976, 72, 9, 2, 40, 11),        # three column blocks, six chunks a wave
    (5456, 40, 4, 1, 0, 6),          # two column blocks, eleven chunks a wave
    (4096, 1792, 8, 2, 0, 8),        # Mixtral-wide rows, the T * d limit
    (3584, 2560, 16, 8, 4104, 3),    # fine-grained experts and a shared one of several groups
    (8192, 136, 5, 2, 0, 4),         # the widest rows
    (128, 64, 256, 16, 0, 16),       # most experts, most ranks
    (136, 64, 200, 1, 0, 5),
]


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
@pytest.mark.parametrize("d,f,n,k,fs,T", SHAPES)
def test_layer_against_its_definition(d, f, n, k, fs, T, act):
    torch = torch_cuda()
    say("layer_tokens", d, f, n, k, fs, T, act)
    layer = Layer(torch, d * 7 + f + T, d, f, n, k, fs)
    dtype = getattr(torch, act)
    check(layer, states(torch, T, T, d, dtype), None, "plain")
    check(layer, states(torch, T + 100, T, d, dtype), states(torch, 5, T, d, dtype), "with y_in")


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
@pytest.mark.parametrize("d,f,n,k,fs,T", [
    # up to 8 logits and rows of 2048: routed inside gate/up
    (2048, 264, 8, 2, 0, 1),
    (2040, 72, 4, 4, 0, 2),          # ends inside a chunk
    (1544, 136, 2, 1, 0, 4),         # rows of four chunks a wave, the last waves short
    (1536, 136, 1, 1, 24, 5),        # the columns fill the rings; one expert
    (520, 64, 1, 1, 16, 8),          # bf16: eight columns; fp32: two column blocks
    (256, 4104, 3, 2, 40960, 1),     # a shared expert that fills the rings before the routing
    (2056, 264, 8, 2, 0, 1),         # just beyond
    (512, 264, 9, 2, 0, 1),
])
def test_the_smallest_calls(d, f, n, k, fs, T, act):
    torch = torch_cuda()
    say("layer_tokens small", d, f, n, k, fs, T, act)
    layer = Layer(torch, d * 5 + f + T, d, f, n, k, fs)
    dtype = getattr(torch, act)
    check(layer, states(torch, T, T, d, dtype), states(torch, 5, T, d, dtype), "with y_in")
    x = states(torch, T + 9, T, d, dtype)
    x[0, d // 2] = float("nan")
    y, _, _ = layer.run(x)
    assert torch.isnan(y[0]).all()
    clean = x.clone()
    clean[0, d // 2] = 0.0
    ref, _, _ = layer.run(clean)
    if T > 1:
        got, want = y[1:].double(), ref[1:].double()
        rms = want.pow(2).mean(1, keepdim=True).sqrt()
        # the batch's experts, and with them the groups of the sums, may differ
        tol = 16 * 2.0 ** -24 * (2 * d ** 0.5 + (k * f + fs) ** 0.5) * rms
        if act == "bfloat16":
            tol = tol + 2.0 ** -16 * 8 * rms + 2.0 ** -7 * want.abs()
        assert bool(((got - want).abs() <= tol).all())


def test_full_mixtral_layer():
    torch = torch_cuda()
    say("layer_tokens mixtral")
    layer = Layer(torch, 3, 4096, 14336, 8, 2)
    for T in (1, 8):
        check(layer, states(torch, T, T, 4096, torch.float32), None, f"T={T}")


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
def test_experts_without_a_slot(act):
    """Slots permuted, absent (-1) and out of range: those experts add nothing."""
    torch = torch_cuda()
    say("layer_tokens slots", act)
    dtype = getattr(torch, act)
    slots = [3, -1, 0, 9, 1, -5, 2, 99]
    layer = Layer(torch, 8, 320, 200, 8, 3, 0, slots)
    layer.nslots = 4
    check(layer, states(torch, 2, 7, 320, dtype), None, "some absent")
    # none present: y_in, or zeros
    none = Layer(torch, 9, 320, 200, 8, 3, 0, [-1] * 8)
    x, y_in = states(torch, 3, 7, 320, dtype), states(torch, 4, 7, 320, dtype)
    y, _, _ = none.run(x)
    assert torch.all(y == 0)
    y, _, _ = none.run(x, y_in)
    assert torch.equal(y, y_in)
    # none present beside a shared expert
    check(Layer(torch, 10, 320, 200, 8, 3, 136, [-1] * 8), x, y_in, "shared alone")


def test_in_place_and_neighbours():
    """y over y_in gives the same; nothing behind the last row is written."""
    torch = torch_cuda()
    say("layer_tokens in place")
    layer = Layer(torch, 11, 264, 264, 6, 2, 72)
    x, y_in = states(torch, 1, 5, 264, torch.float32), states(torch, 2, 5, 264, torch.float32)
    y, _, _ = layer.run(x, y_in)
    buf = torch.full((7, 264), 123.0, device="cuda")
    buf[:5] = y_in
    layer.call(x, buf[:5], layer.workspace(5), y_in=buf[:5])
    assert torch.equal(buf[:5], y) and torch.all(buf[5:] == 123.0)


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
@pytest.mark.parametrize("d,n,T,fs", [(264, 6, 5, 72), (1024, 4, 2, 0), (4096, 8, 8, 0), (256, 2, 1, 2056)])
def test_residual_over_its_own_input(d, n, T, fs, act):
    """x as y_in, and y over both: a residual layer that keeps its states in one buffer."""
    torch = torch_cuda()
    say("layer_tokens over x", d, n, T, fs, act)
    layer = Layer(torch, 30 + d, d, 520, n, 2, fs)
    x = states(torch, 3, T, d, getattr(torch, act))
    y, _, _ = layer.run(x, x)
    state = x.clone()
    for _ in range(3):
        state.copy_(x)
        layer.call(state, state, layer.workspace(T), y_in=state)
        assert torch.equal(state, y)


def test_ties_and_a_token_of_nan():
    """Equal logits go to the lower ids; a token of NaN or infinities leaves the others alone."""
    torch = torch_cuda()
    say("layer_tokens ties, NaN")
    d, n = 256, 20
    layer = Layer(torch, 12, d, 136, n, 4, 0, wr=torch.zeros((n, d)))
    x = states(torch, 5, 6, d, torch.float32)
    y, idx, w = layer.run(x)
    assert np.array_equal(idx, np.tile(np.arange(4), (6, 1))) and np.all(w == 0.25)
    layer = Layer(torch, 13, d, 136, n, 4, 72)
    for dtype in (torch.float32, torch.bfloat16):
        x = states(torch, 6, 6, d, dtype)
        ey, _, _, cols = layer.expect(x)
        for bad in (float("nan"), float("inf"), -float("inf")):
            z = x.clone()
            z[2, 17] = bad
            y, idx, _ = layer.run(z)
            # (not bit for bit: which experts the batch selects, and with it how the hidden
            # columns are grouped into fp32 sums, has changed with the token)
            keep = [0, 1, 3, 4, 5]
            close(layer, y[keep], ey[keep], cols[keep], f"beside {bad}")
            assert torch.all(torch.isnan(y[2])) and np.all((idx >= 0) & (idx < n))


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
def test_an_expert_of_nan_reaches_its_own_tokens_only(act):
    torch = torch_cuda()
    say("layer_tokens NaN expert", act)
    d, f, n, k, T = 256, 136, 12, 2, 9
    layer = Layer(torch, 21, d, f, n, k, 72)
    x = states(torch, 11, T, d, getattr(torch, act))
    ey, idx, _, cols = layer.expect(x)
    for part in (0, f * d, 2 * f * d):                   # W1, W3, W2
        for bad in (float("nan"), float("inf")):
            e = int(idx[0, 0])
            keep = layer.pool[e].clone()
            layer.pool[e, part:part + f * d] = bad
            y, _, _ = layer.run(x)
            layer.pool[e] = keep
            for t in range(T):
                if e in idx[t]:
                    assert not torch.any(torch.isfinite(y[t])), t
                else:
                    close(layer, y[t:t + 1], ey[t:t + 1], cols[t:t + 1], f"t={t} beside an expert of {bad}")


def test_large_and_small_values():
    """Values near the top of the fp32 range stay finite in the products' parts, tiny ones keep
    their precision (the three parts are exact down to 2^-110)."""
    torch = torch_cuda()
    say("layer_tokens ranges")
    d, f = 128, 64
    layer = Layer(torch, 14, d, f, 4, 2)
    x = states(torch, 7, 4, d, torch.float32)
    for scale in (2.0 ** -40, 2.0 ** 30):
        check(layer, x * scale, None, f"scale {scale}")


@pytest.mark.parametrize("T,n", [(4, 8), (1, 8)])   # three launches, and two
def test_captured_and_replayed(T, n):
    """The call in a graph, replayed between eager calls on the same workspace's twin."""
    torch = torch_cuda()
    say("layer_tokens graph")
    layer = Layer(torch, 15, 512, 520, n, 2, 136)
    x = states(torch, 8, T, 512, torch.float32)
    y, ws = torch.empty_like(x), layer.workspace(T)
    graph = capture(torch, lambda: layer.call(x, y, ws))
    for i in range(4):
        x.copy_(states(torch, 20 + i, T, 512, torch.float32))
        graph.replay()
        eager, _, _ = layer.run(x)
        torch.cuda.synchronize()
        assert torch.equal(y, eager), i


def test_two_streams_at_once():
    """Two layers on two streams, each with its workspace, give what they give alone."""
    torch = torch_cuda()
    say("layer_tokens two streams")
    layers = [Layer(torch, 30 + i, 1024, 1024 + 8 * i, 8, 2) for i in range(2)]
    x = states(torch, 9, 8, 1024, torch.float32)
    alone = [l.run(x)[0] for l in layers]
    streams = side_streams(torch)[:2]
    ws = [l.workspace(8) for l in layers]
    ys = [[torch.empty_like(x) for _ in range(5)] for _ in range(2)]
    torch.cuda.synchronize()
    for r in range(5):
        for i in range(2):
            layers[i].call(x, ys[i][r], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for r in range(5):
            assert torch.equal(ys[i][r], alone[i]), (i, r)


def test_against_the_calls_it_replaces():
    """The same layer through router_topk and expert_ffn_tokens."""
    torch = torch_cuda()
    say("layer_tokens against router_topk + expert_ffn_tokens")
    d, f, n, k, T = 1024, 1032, 8, 2, 6
    layer = Layer(torch, 16, d, f, n, k)
    x = states(torch, 10, T, d, torch.float32)
    y, idx, w = layer.run(x)
    ridx, rw = moe.router_topk(x, layer.wr, k)
    ref = torch.empty_like(x)
    ws = torch.empty(moe.ffn_tokens_workspace_bytes(T, k, d, f), dtype=torch.uint8, device="cuda")
    moe.expert_ffn_tokens(x, layer.pool, n, ridx, rw, d, f, ref, ws)
    torch.cuda.synchronize()
    assert np.array_equal(idx, ridx.cpu().numpy()) and np.allclose(w, rw.cpu().numpy(), rtol=2e-7, atol=0)
    err = (y - ref).abs().max() / ref.pow(2).mean().sqrt()
    assert float(err) <= 2.0 ** -16 * 4     # the other path keeps activations to 2^-18, twice


def test_arguments():
    """Tensors the kernels could not read as they are refused by name; no tokens are no call."""
    torch = torch_cuda()
    say("layer_tokens arguments")
    layer = Layer(torch, 17, 64, 64, 4, 2, 64)
    x = states(torch, 1, 3, 64, torch.float32)
    y, ws = torch.empty_like(x), layer.workspace(3)
    good = dict(x=x, w_router=layer.wr, slot_pool=layer.pool, f=64, k=2, y=y, workspace=ws, shared=layer.shared, f_shared=64)
    moe.layer_tokens(**good)
    bad = [("x", dict(x=torch.zeros((3, 128), device="cuda")[:, ::2])), ("y", dict(y=y.bfloat16())), ("y", dict(y=y[:2])),
           ("y_in", dict(y_in=y.cpu())), ("w_router", dict(w_router=layer.wr.double())), ("slot_pool", dict(slot_pool=layer.pool[:3])),
           ("slotmap", dict(slotmap=torch.zeros(3, dtype=torch.int32, device="cuda"))), ("shared", dict(shared=None)),
           ("shared", dict(shared=layer.shared[:-128])), ("idx", dict(idx=torch.zeros((3, 2), device="cuda"))),
           ("w", dict(w=torch.zeros((2, 3), device="cuda"))), ("workspace", dict(workspace=ws.cpu()))]
    for name, change in bad:
        with pytest.raises(ValueError, match=f"layer_tokens: {name} must"):
            moe.layer_tokens(**{**good, **change})
    with pytest.raises(moe.MoeError, match="workspace"):
        moe.layer_tokens(**{**good, "workspace": ws[:256]})
    none = torch.empty((0, 64), device="cuda")
    moe.layer_tokens(none, layer.wr, layer.pool, 64, 2, none, ws[:0], shared=layer.shared, f_shared=64)
