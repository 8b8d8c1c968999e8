"""GPU tests of moe_adapter_project (low-rank adapters of many requests beside a projection they
share) against its definition in 64 bits: y = y_in + W x + scale B (A x), each token's own A, B.

Tolerance. Products are exact (bf16 weights, fp32 activations and low-rank values in three bf16
parts) and sums fp32: a sum of K terms of random sign is off by about sqrt(K) roundings of its
size, 2^-24 each. The base takes one such sum (K = d_in), the adapter's part two (d_in, rank).
With a factor 8 for the largest of some thousand outputs: 8 * 2^-24 * (2 sqrt(d_in) + sqrt(rank)
+ 1) of the RMS of |y_in| + |W x| + |scale B A x|. Beside bf16 activations the low-rank values of
long batches have two parts (2^-17 relative), and y is rounded once, by at most 2^-8 of its value."""
import numpy as np
import pytest

from _gpu_util import capture, say, side_streams, torch_cuda

pytestmark = pytest.mark.gpu

import paper_2512_16473_amd as moe  # noqa: E402


class Case:
    def __init__(self, torch, seed, T, d, o, r, n, act, spread="each", w=True, scale=True, y_in=False, pad=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.torch = torch
        dtype = getattr(torch, act)
        def normal(std, *shape):
            return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)
        self.T, self.d, self.o, self.r, self.n, self.dtype = T, d, o, r, n, dtype
        self.x = normal(1.0, T, d + pad)[:, :d].to(dtype) if not pad else normal(1.0, T, d + pad).to(dtype)[:, :d]
        self.w = normal(d ** -0.5, o, d).bfloat16() if w else None
        self.a = normal(d ** -0.5, n, r, d).bfloat16()
        self.b = normal(r ** -0.5, n, o, r).bfloat16()
        self.scale = torch.empty(n, device="cuda").uniform_(0.25, 2.0, generator=g) if scale else None
        self.y_in = normal(1.0, T, o + pad).to(dtype)[:, :o] if y_in else None
        u = torch.empty(T, device="cuda").uniform_(generator=g)
        if spread == "each":
            self.ids = ((u * (n + 2)).int() - 1).contiguous()            # -1 and n: none
        elif spread == "one":
            self.ids = torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
        elif spread == "none":
            self.ids = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        else:
            self.ids = (torch.arange(T, device="cuda") * (n + 1) // T - 1).int().contiguous()

    def workspace(self):
        nbytes = moe.adapter_workspace_bytes(self.T, self.d, self.o, self.r, self.dtype)
        return self.torch.full((nbytes,), 0xFF, dtype=self.torch.uint8, device="cuda")   # any content

    def call(self, y, ws, y_in=None, stream=None):
        return moe.adapter_project(self.x, self.w, self.a, self.b, self.ids, y, ws, scale=self.scale,
                                   y_in=self.y_in if y_in is None else y_in, stream=stream)

    def run(self, pad=0):
        buf = self.torch.full((self.T + 2, self.o + pad), 77.0, dtype=self.dtype, device="cuda")
        y = buf[:self.T, :self.o]
        self.call(y, self.workspace())
        self.torch.cuda.synchronize()
        assert self.torch.all(buf[self.T:] == 77.0) and self.torch.all(buf[:, self.o:] == 77.0)
        return y

    def expect(self):
        torch = self.torch
        x = self.x.double()
        zero = torch.zeros((self.T, self.o), dtype=torch.float64, device="cuda")
        base = x @ self.w.double().t() if self.w is not None else zero
        low = zero.clone()
        for i in range(self.n):
            m = (self.ids == i).nonzero()[:, 0]
            s = 1.0 if self.scale is None else float(self.scale[i])
            low[m] = s * (x[m] @ self.a[i].double().t()) @ self.b[i].double().t()
        y_in = self.y_in.double() if self.y_in is not None else zero
        return y_in + base + low, y_in.abs() + base.abs() + low.abs()

    def close(self, y, what=""):
        ey, size = self.expect()
        rms = (size ** 2).mean(1, keepdim=True).sqrt()
        tol = 8 * 2.0 ** -24 * (2 * self.d ** 0.5 + self.r ** 0.5 + 1) * rms
        if self.dtype == self.torch.bfloat16:
            tol = tol + 8 * 2.0 ** -17 * rms + 2.0 ** -8 * ey.abs()
        worst = float(((y.double() - ey).abs() / tol.clamp_min(1e-300)).max())
        assert worst <= 1.0, f"{what}: {worst:.2f} x the tolerance"


ACTS = ["float32", "bfloat16"]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,d,o,r,n,spread", [
    (1, 256, 512, 8, 4, "one"),        # the smallest call
    (1, 8, 8, 8, 1, "one"),            # one short row block, one piece of a chunk
    (3, 264, 520, 16, 5, "each"),      # ends inside a chunk and a row block
    (5, 4096, 1032, 24, 3, "each"),    # one group of eight full units
    (6, 72, 4104, 64, 9, "each"),      # two column blocks of fp32, two chunks
    (8, 4104, 264, 40, 40, "each"),    # two groups
    (11, 5000, 136, 128, 4, "each"),   # three column blocks, the largest rank
    (16, 14336, 512, 64, 32, "each"),  # groups, most tokens of the streamed form
    (16, 1024, 1024, 16, 2, "none"),
    (16, 136, 264, 16, 300, "each"),
])
def test_decode_batches(T, d, o, r, n, spread, act):
    torch = torch_cuda()
    say("adapter", T, d, o, r, n, spread, act)
    c = Case(torch, T + d, T, d, o, r, n, act, spread)
    c.close(c.run(), "plain")
    c = Case(torch, T + d + 1, T, d, o, r, n, act, spread, y_in=True, scale=False, pad=24)
    c.close(c.run(pad=8), "strides, y_in, no scale")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,d,o,r,n,spread", [
    (17, 8, 8, 8, 2, "each"),            # least of everything
    (17, 4096, 264, 16, 30, "each"),     # one block of 32 rows, split over K
    (40, 2056, 136, 32, 9, "each"),      # the last 16 tokens begin among the ones before
    (64, 264, 520, 24, 7, "runs"),       # padded K steps
    (97, 1024, 2048, 128, 3, "each"),    # two K steps of ranks
    (160, 576, 776, 64, 5, "runs"),
    (256, 640, 256, 72, 256, "each"),    # a full tile, most adapters in one
    (300, 3592, 1288, 40, 6, "runs"),    # two tiles of tokens
    (700, 1032, 3000, 8, 4, "one"),
    (1024, 192, 4096, 32, 2, "none"),
    (2050, 512, 9000, 16, 11, "runs"),   # more tiles than work groups: whole and split ones
])
def test_long_batches(T, d, o, r, n, spread, act):
    torch = torch_cuda()
    say("adapter", T, d, o, r, n, spread, act)
    c = Case(torch, T + d, T, d, o, r, n, act, spread)
    c.close(c.run(), "plain")
    c = Case(torch, T + d + 1, T, d, o, r, n, act, spread, y_in=True, scale=False, pad=40)
    c.close(c.run(pad=16), "strides, y_in, no scale")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [1, 16, 17, 270])
def test_adapters_alone(T, act):
    """No W: the adapters' part (and y_in) only."""
    torch = torch_cuda()
    say("adapter alone", T, act)
    for y_in in (False, True):
        c = Case(torch, T, T, 520, 776, 24, 5, act, "each", w=False, y_in=y_in)
        c.close(c.run(), f"y_in={y_in}")
    c = Case(torch, T, T, 520, 776, 24, 5, act, "none", w=False, y_in=True)
    assert torch.equal(c.run(), c.y_in)
    c = Case(torch, T, T, 520, 776, 24, 5, act, "none", w=False)
    assert torch.all(c.run() == 0)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [7, 40])
def test_no_adapters_held(T, act):
    torch = torch_cuda()
    say("adapter n = 0", T, act)
    c = Case(torch, T, T, 264, 136, 8, 1, act, "none")
    c.n, c.a, c.b, c.scale = 0, c.a[:0], c.b[:0], None
    c.close(c.run(), "n = 0")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [9, 200])
def test_in_place_and_a_token_of_nan(T, act):
    """y over y_in gives the same bits; a token of NaN or infinities leaves the others' alone."""
    torch = torch_cuda()
    say("adapter in place, NaN", T, act)
    c = Case(torch, T, T, 328, 264, 16, 4, act, "each", y_in=True)
    y = c.run()
    z = c.y_in.clone()
    c.call(z, c.workspace(), y_in=z)
    assert torch.equal(y, z)
    keep = [t for t in range(T) if t != 4]
    for bad in (float("nan"), float("inf"), -float("inf")):
        c.x = c.x.clone()
        c.x[4, 5] = bad
        z = c.run()
        assert torch.equal(z[keep], y[keep])
        assert not torch.any(torch.isfinite(z[4]))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T", [9, 200])
def test_an_adapter_of_nan_reaches_its_own_tokens_only(T, act):
    torch = torch_cuda()
    say("adapter of NaN", T, act)
    c = Case(torch, T + 50, T, 328, 264, 16, 4, act, "each", y_in=True)
    y = c.run()
    mine = c.ids == 2
    assert 0 < int(mine.sum()) < T
    for name in ("a", "b"):
        for bad in (float("nan"), float("inf")):
            was = getattr(c, name)
            broken = was.clone()
            broken[2] = bad
            setattr(c, name, broken)
            z = c.run()
            setattr(c, name, was)
            assert torch.equal(z[~mine], y[~mine])
            assert not torch.any(torch.isfinite(z[mine]))


@pytest.mark.parametrize("T", [8, 100])
def test_captured_and_replayed(T):
    torch = torch_cuda()
    say("adapter graph", T)
    c = Case(torch, 3, T, 1032, 1288, 16, 6, "bfloat16", "each")
    y, ws = torch.empty((T, c.o), dtype=c.dtype, device="cuda"), c.workspace()
    graph = capture(torch, lambda: c.call(y, ws))
    for i in range(4):
        c.x.copy_(torch.randn(c.x.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(i)).to(c.dtype))
        c.ids.copy_((c.ids + 2) % 7 - 1)
        graph.replay()
        eager = c.run()
        assert torch.equal(y, eager), i


@pytest.mark.parametrize("T", [8, 300])
def test_two_streams_at_once(T):
    torch = torch_cuda()
    say("adapter two streams", T)
    cases = [Case(torch, 5 + i, T, 2056, 1288 + 512 * i, 16, 6, "bfloat16", "each") for i in range(2)]
    alone = [c.run() for c in cases]
    streams = side_streams(torch)[:2]
    ws = [c.workspace() for c in cases]
    ys = [[torch.empty((T, c.o), dtype=c.dtype, device="cuda") for _ in range(5)] for c in cases]
    torch.cuda.synchronize()
    for r in range(5):
        for i in range(2):
            cases[i].call(ys[i][r], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for r in range(5):
            assert torch.equal(ys[i][r], alone[i]), (i, r)


def test_offsets_beyond_32_bits():
    """Adapters and rows that lie more than 4 GiB into their tensors."""
    torch = torch_cuda()
    say("adapter far offsets")
    n, r, d, o = 300, 128, 57344, 264         # A: 300 * 14.7 MB
    a = torch.zeros((n, r, d), dtype=torch.bfloat16, device="cuda")
    for T in (3, 20):
        c = Case(torch, T, T, d, o, r, 1, "bfloat16", "one")
        a[n - 1] = c.a[0]
        b = torch.zeros((n, o, r), dtype=torch.bfloat16, device="cuda")
        b[n - 1] = c.b[0]
        y = c.run()
        s = torch.ones(n, device="cuda")
        s[n - 1] = c.scale[0]
        c2 = Case(torch, T, T, d, o, r, 1, "bfloat16", "one")
        c2.a, c2.b, c2.scale, c2.ids = a, b, s, torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
        assert torch.equal(c2.run(), y)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,r,n,spread", [
    (65536, 8, 3, "each"),     # the most tokens of a call
    (65536, 8, 300, "runs"),
    (300, 128, 40, "each"),    # more adapters in a tile than fit beside their v, twice 64 ranks
    (300, 72, 40, "runs"),     # the second 64 ranks end early
])
def test_many_tokens_and_many_adapters(T, r, n, spread, act):
    say(f"adapter {T} tokens r={r} n={n} {spread} {act}")
    c = Case(torch_cuda(), 71 + T + n, T, 200, 296, r, n, act, spread=spread, y_in=True)
    c.close(c.run(), f"{T} tokens, {n} adapters")


def test_arguments():
    """Tensors the kernels could not read as they are refused by name; no tokens are no call."""
    torch = torch_cuda()
    say("adapter arguments")
    c = Case(torch, 1, 5, 64, 128, 8, 3, "bfloat16")
    y = torch.empty((5, 128), dtype=torch.bfloat16, device="cuda")
    good = dict(x=c.x, w=c.w, a=c.a, b=c.b, adapters=c.ids, y=y, workspace=c.workspace(), scale=c.scale)
    moe.adapter_project(**good)
    wide = torch.zeros((5, 256), dtype=torch.bfloat16, device="cuda")
    bad = [("x", dict(x=wide[:, :128:2])), ("y", dict(y=y.float())), ("y", dict(y=wide[:, ::2])), ("y_in", dict(y_in=y[:4])),
           ("w", dict(w=c.w.float())), ("w", dict(w=c.w.t())), ("b", dict(b=c.b[:2])), ("a", dict(a=c.a.transpose(0, 1))),
           ("adapters", dict(adapters=c.ids.long())), ("scale", dict(scale=c.scale[:2])),
           ("workspace", dict(workspace=torch.empty(8, dtype=torch.uint8)))]
    for name, change in bad:
        with pytest.raises(ValueError, match=f"adapter_project: {name} must"):
            moe.adapter_project(**{**good, **change})
    with pytest.raises(moe.MoeError, match="x_stride=76"):
        moe.adapter_project(**{**good, "x": torch.zeros((5, 76), dtype=torch.bfloat16, device="cuda")[:, :64]})
    with pytest.raises(moe.MoeError, match="workspace"):
        moe.adapter_project(**{**good, "workspace": good["workspace"][:256]})
    none = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    moe.adapter_project(none, c.w, c.a, c.b, c.ids[:0], y[:0], good["workspace"][:0])
    moe.adapter_project(none, c.w, c.a, c.b, c.ids[:0], y[:0], None)


def test_a_batch_through_the_layer_and_its_adapted_shared_expert():
    """One decode step: the routed experts by layer_tokens, the shared expert's three projections
    by adapter_project straight out of its slab, each request with its adapters, the second on top
    of the first through y_in."""
    torch = torch_cuda()
    say("layer_tokens + adapter_project")
    d, f, n, k, fs, T, na, r = 1024, 520, 16, 4, 1288, 7, 5, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(77)
    def normal(std, *shape):
        return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g)
    x = normal(1.0, T, d)
    wr, pool = normal(d ** -0.5, n, d), normal(d ** -0.5, n, moe.slab_bytes(d, f) // 2).bfloat16()
    slab = normal(d ** -0.5, 3 * d * fs).bfloat16()
    w1, w3, w2 = slab[:fs * d].view(fs, d), slab[fs * d:2 * fs * d].view(fs, d), slab[2 * fs * d:].view(d, fs)
    ids = torch.tensor([0, 3, -1, 3, 1, 4, 0], dtype=torch.int32, device="cuda")
    ad = [(normal(i ** -0.5, na, r, i).bfloat16(), normal(0.5 * r ** -0.5, na, q, r).bfloat16())
          for i, q in ((d, fs), (d, fs), (fs, d))]

    def project(src, w, ab, dst, y_in=None):
        ws = torch.empty(moe.adapter_workspace_bytes(T, src.shape[1], w.shape[0], r, src.dtype), dtype=torch.uint8, device="cuda")
        return moe.adapter_project(src, w, ab[0], ab[1], ids, dst, ws, y_in=y_in)

    y = torch.empty_like(x)
    ws = torch.empty(moe.layer_tokens_workspace_bytes(T, d, f, n, k), dtype=torch.uint8, device="cuda")
    idx = torch.empty((T, k), dtype=torch.int32, device="cuda")
    gw = torch.empty((T, k), device="cuda")
    moe.layer_tokens(x, wr, pool, f, k, y, ws, idx=idx, w=gw)
    gate, up = torch.empty((T, fs), device="cuda"), torch.empty((T, fs), device="cuda")
    project(x, w1, ad[0], gate)
    project(x, w3, ad[1], up)
    h = torch.nn.functional.silu(gate) * up
    project(h, w2, ad[2], y, y_in=y)
    torch.cuda.synchronize()

    xd = x.double()
    ref = torch.zeros((T, d), dtype=torch.float64, device="cuda")
    for t in range(T):
        for e, q in zip(idx[t].tolist(), gw[t].tolist()):
            m = pool[e, :3 * d * f].double()
            a = m[:f * d].view(f, d) @ xd[t]
            ref[t] += q * (m[2 * f * d:].view(d, f) @ (a * torch.sigmoid(a) * (m[f * d:2 * f * d].view(f, d) @ xd[t])))
        def proj(v, w, ab):
            o = w.double() @ v
            i = int(ids[t])
            return o if i < 0 else o + ab[1][i].double() @ (ab[0][i].double() @ v)
        a = proj(xd[t], w1, ad[0])
        ref[t] += proj(a * torch.sigmoid(a) * proj(xd[t], w3, ad[1]), w2, ad[2])
    rms = ref.pow(2).mean(1, keepdim=True).sqrt()
    # fp32 sums of 1024 and 1288 terms, twice over: as in the two operators' own tests
    tol = 8 * 2.0 ** -24 * (4 * d ** 0.5 + 2 * fs ** 0.5 + (k * f) ** 0.5 + 3 * r ** 0.5) * rms
    assert torch.all((y.double() - ref).abs() <= tol)
