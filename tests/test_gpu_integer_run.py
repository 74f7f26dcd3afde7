"""The integer rows, their product, the norms, the 8-bit cache and its attention as a block runs them: each step held to its 64-bit
reference on the operands that it was given, the steps recorded and replayed, and products in every tile."""
import numpy as np
import pytest
import torch

from oracle import integer as ref
from oracle import scaled
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_cache import check_attention
from tests.test_gpu_integer import gelu_err
from tests.test_gpu_scaled import U8, U32, UB, bf16, count, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


class Block:
    """A block of hidden size heads * dh with sandwich norms: weights as integers laid out once, buffers for `rows` rows of
    the tokens, and its steps in order."""

    def __init__(self, rows, tokens, heads, kv_heads, dh, F, q_len, k_len, dims, seed=0):
        rng = np.random.default_rng([seed, rows, dh])
        self.rows, self.heads, self.kv, self.dh, self.D, self.F = rows, heads, kv_heads, dh, heads * dh, F
        self.cu, self.off = (np.concatenate([[0], np.cumsum(v)]).astype(np.int32) for v in (q_len, k_len))
        B, D = len(q_len), self.D
        idx = np.concatenate([o + np.sort(rng.permutation(k)[:n]) for o, n, k in zip(self.off, q_len, k_len)]).astype(np.int32)
        self.idx = np.concatenate([idx, np.zeros(rows - len(idx), np.int32)])
        self.m, self.live = count(len(idx)), len(idx)
        self.d_cu, self.d_off, self.d_idx = dev(self.cu), dev(self.off), dev(self.idx)
        self.coord = dev(rng.integers(0, 200, (tokens, len(dims))).astype(np.int32))
        self.rope, self.dims = fdl.rope_axes(dims), dims
        self.mod = dev((0.3 * rng.standard_normal((B, 6 * D))).astype(np.float32))
        self.norms = [dev((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)) for _ in range(4)]
        self.w = {}
        for name, n, k in (("qkv", (heads + 2 * kv_heads) * dh, D), ("o", D, D), ("1", F, D), ("2", D, F)):
            q, s = torch.empty((n, k), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
            fdl.fd_int_rows(bf16(rng.standard_normal((n, k)) / np.sqrt(k)).cuda(), q, s)
            self.w[name] = (q, s, dev((0.02 * rng.standard_normal(n)).astype(np.float32)))
        self.h = dev(rng.standard_normal((rows, D)).astype(np.float32))
        r16 = lambda n: torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.a, self.sa = torch.zeros((rows, D), dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
        self.g, self.sg = torch.zeros((rows, F), dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
        self.qkv, self.q, self.o, self.y, self.f = r16((heads + 2 * kv_heads) * dh), r16(D), r16(D), r16(D), r16(F)
        old = lambda: ref.head_codes(rng.standard_normal((tokens, kv_heads, dh)))  # noqa: E731
        (k, ks), (v, vs) = old(), old()
        self.k, self.ks, self.v, self.vs = dev(k.reshape(tokens, -1)), dev(ks.T), dev(v.reshape(tokens, -1)), dev(vs.T)
        self.ws = torch.empty(fdl.fd_cache_attention_ws_size(rows, heads, kv_heads, dh), dtype=torch.uint8, device="cuda")

    def part(self, i):
        return self.mod[:, i * self.D:(i + 1) * self.D]

    def product(self, a, sa, name, y, gelu=False):
        w, sw, bias = self.w[name]
        fdl.fd_int_linear(a, sa, w, sw, y, bias=bias, gelu=gelu, m=self.m)

    def steps(self):
        """(name, call) of the block's steps."""
        n = self.norms
        norm = lambda to, **kw: fdl.fd_norm_residual(self.h, to, self.d_cu, self.m, a_scale=self.sa if to is not None else None, **kw)  # noqa: E731
        return [
            ("norm1", lambda: norm(self.a, weight=n[0], shift=self.part(0), mod_scale=self.part(1))),
            ("qkv", lambda: self.product(self.a, self.sa, "qkv", self.qkv)),
            ("cache", lambda: fdl.fd_cache_write(self.qkv, self.coord, self.d_idx, self.m, self.q, self.k, self.ks, self.v, self.vs, self.heads, self.kv,
                                                 self.dh, rope=self.rope)),
            ("attention", lambda: fdl.fd_cache_attention(self.q, self.k, self.ks, self.v, self.vs, self.o, self.d_cu, self.d_off, self.heads, self.kv, self.dh, self.ws)),
            ("rows_o", lambda: fdl.fd_int_rows(self.o, self.a, self.sa, m=self.m)),
            ("o", lambda: self.product(self.a, self.sa, "o", self.y)),
            ("norm2", lambda: norm(self.a, y=self.y, post_weight=n[1], gate=self.part(2), residual=0.875, weight=n[2], shift=self.part(3), mod_scale=self.part(4))),
            ("mlp1", lambda: self.product(self.a, self.sa, "1", self.f, gelu=True)),
            ("rows_f", lambda: fdl.fd_int_rows(self.f, self.g, self.sg, m=self.m)),
            ("mlp2", lambda: self.product(self.g, self.sg, "2", self.y)),
            ("residual", lambda: norm(None, y=self.y, post_weight=n[3], gate=self.part(5), residual=0.875)),
        ]

    def state(self):
        return {k: getattr(self, k) for k in ("h", "a", "sa", "qkv", "q", "k", "ks", "v", "vs", "o", "y", "f", "g", "sg")}


BLOCKS = {
    "image": lambda: Block(200, 400, 6, 2, 64, 1088, [100, 0, 37], [250, 50, 100], [32, 32]),
    "video": lambda: Block(700, 1500, 4, 4, 128, 1024, [650], [1500], [44, 42, 42]),
    "tiny": lambda: Block(5, 9, 4, 4, 16, 64, [2, 3], [4, 5], [8, 8]),
}


def num(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("name", list(BLOCKS))
def test_block(name):
    """One block, step by step: each result against the 64-bit reference of the operands that the step had in memory, within the bounds of
    the operators' own tests.  (A 64-bit chain beside it would show less: a value next to a rounding's limit that one side rounds
    up and the other down differs by a whole step of 8 bits.)"""
    b = BLOCKS[name]()
    M, D = b.live, b.D
    of_row = np.repeat(np.arange(len(b.cu) - 1), np.diff(b.cu))
    mod = num(b.mod)
    pick = lambda i: mod[of_row, i * D:(i + 1) * D]  # noqa: E731
    for step, call in b.steps():
        gh.say(f"{name}: {step}")
        before = {k: num(t)[:M] if t.dtype != torch.uint8 else t.cpu().numpy() for k, t in b.state().items()}
        call()
        torch.cuda.synchronize()
        after = {k: num(t)[:M] if t.dtype != torch.uint8 else t.cpu().numpy() for k, t in b.state().items()}
        if step in ("norm1", "norm2", "residual"):
            y = None if step == "norm1" else before["y"]
            post, gate = {"norm1": (None, None), "norm2": (num(b.norms[1]), pick(2)), "residual": (num(b.norms[3]), pick(5))}[step]
            w, s, t = {"norm1": (num(b.norms[0]), pick(1), pick(0)), "norm2": (num(b.norms[2]), pick(4), pick(3)), "residual": (None, None, None)}[step]
            wh, add, wa = ref.norm_residual(before["h"], y, post, gate, 0.875, w, t, s, 1e-6)
            h_err = 2 * U32 * (np.abs(wh) + np.abs(before["h"])) + 40 * U32 * np.abs(add)
            assert np.all(np.abs(after["h"] - wh) <= h_err)
            if step == "residual":
                continue
            # the norm of the h in memory, so its own error is not counted
            wa = ref.norm_residual(after["h"], None, None, None, 1.0, w, t, s, 1e-6)[2]
            sa, q = after["sa"][:, None], after["a"]
            err = 40 * U32 * (np.abs(wa) + np.abs(t)) + 40 * U32 * np.abs(t)
            assert np.all(np.abs(q * sa - wa) <= sa * (0.5 + 127 * 3 * U32) + err) and np.all(np.max(np.abs(q), 1) == 127)
        elif step in ("qkv", "o", "mlp1", "mlp2"):
            a, sa, out, key = {"qkv": ("a", "sa", "qkv", "qkv"), "o": ("a", "sa", "y", "o"), "mlp1": ("a", "sa", "f", "1"), "mlp2": ("g", "sg", "y", "2")}[step]
            w, sw, bias = (t.cpu().numpy() for t in b.w[key])
            z, size = ref.linear(before[a], before[sa], w, sw, bias)
            err, want = 4 * U32 * size + U32 * np.abs(z), z
            if step == "mlp1":
                want, err = scaled.gelu(z), 1.13 * err + gelu_err(z)
            assert np.all(np.abs(after[out] - want) <= err + UB * (np.abs(want) + err))
        elif step in ("rows_o", "rows_f"):
            x, q, s = ("o", "a", "sa") if step == "rows_o" else ("f", "g", "sg")
            wq, ws = ref.int_rows(before[x])
            np.testing.assert_array_equal(after[q], wq)
            np.testing.assert_array_equal(after[s].astype(np.float32), ws)
        elif step == "cache":
            x = before["qkv"].reshape(M, -1, b.dh)
            qk = scaled.rope(x[:, :b.heads + b.kv], num(b.coord)[b.idx[:M]].astype(np.int64), b.dims, [1e4] * len(b.dims), [1.0] * len(b.dims), False)
            turn = 2.0 ** -20 * np.max(np.abs(qk), 2, keepdims=True)
            assert np.all(np.abs(after["q"].reshape(M, -1, b.dh) - qk[:, :b.heads]) <= turn[:, :b.heads] + UB * (np.abs(qk[:, :b.heads]) + turn[:, :b.heads]))
            for c, s, want, e in (("k", "ks", qk[:, b.heads:], turn[:, b.heads:]), ("v", "vs", x[:, b.heads + b.kv:], 0.0)):
                got = ref.cache_values(after[c].reshape(-1, b.kv, b.dh), after[s])[b.idx[:M]]
                p = scaled.powers(after[s][:, b.idx[:M]].T)[..., None]
                assert np.all(np.abs(got - want) <= np.maximum(U8 * (np.abs(want) + e), 2.0 ** -10 * p) + e)
                others = np.setdiff1d(np.arange(len(after[c])), b.idx[:M])
                assert np.array_equal(after[c][others], before[c][others]) and np.array_equal(after[s][:, others], before[s][:, others])
        else:
            q = b.q[:M].cpu()
            check_attention(after["o"].reshape(M, b.heads, b.dh), q, after["k"], after["ks"], after["v"], after["vs"], b.cu, b.off, b.heads, b.kv, b.dh)
    for t in (b.o, b.y, b.f, b.q, b.qkv):
        assert not t[M:].any()       # rows past the count stay
    assert np.isfinite(num(b.h)).all()


@pytest.mark.parametrize("name", list(BLOCKS))
def test_block_recorded(name):
    """The block's steps recorded into a graph and replayed over several blocks' worth of state, with eager work between: the eager
    block's bits; two graphs, each with its own buffers, one after the other."""
    eager, recs = BLOCKS[name](), [BLOCKS[name]() for _ in range(2)]
    graphs = []
    for r in recs:
        for _, call in BLOCKS[name]().steps():
            call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _, call in r.steps():
                call()
        graphs.append(g)
    for n in range(3):
        for _, call in eager.steps():
            call()
        torch.cuda.synchronize()
        _ = (torch.randn(1 << 14, device="cuda") * 2).sum().item()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for r in recs:
            for (k, a), b in zip(eager.state().items(), r.state().values()):
                assert torch.equal(a, b), f"replay {n}: {k}"


# (M, N, K): 256 x 256 tiles where the host knows the row count: short sums, last blocks of 16 and of 112 columns, tiles that rows
# and columns leave part of, one tile a workgroup and two
# and tiles of split K-blocks: 32 x 32 (from one row to 240; one block and a part, all waves, a last round of some), 32 x 64, 64 x 64
SPLIT = [(1, 4624, 2320), (17, 16, 1296), (33, 528, 1552), (64, 1536, 6144), (240, 1040, 1408), (250, 1040, 4112), (300, 1552, 1296), (500, 1552, 1808), (513, 1536, 2064)]
LARGE = [(8192, 2048, 16), (8190, 2032, 240), (8190, 2048, 512), (14999, 2032, 144)]


@pytest.mark.parametrize("M,N,K", LARGE + SPLIT + [(3000, 1536, 400), (600, 1040, 4112), (129, 4096, 144), (1664, 1536, 1104), (1300, 2064, 400)])
@pytest.mark.parametrize("wide,gelu", [(False, True), (True, False)])
def test_tiles(M, N, K, wide, gelu):
    """Integer operands of few bits, so that the sum times scales of powers of two, and its bias, are exact: every element's place."""
    gh.say(f"tiles {M}x{N}x{K} wide={wide} gelu={gelu}")
    g = torch.Generator(device="cuda")
    g.manual_seed(M + K)
    a, w = (torch.randint(-7, 8, (n, K), generator=g, device="cuda", dtype=torch.int32).to(torch.int8) for n in (M, N))
    sa, sw = (2.0 ** torch.randint(-6, -3, (n,), generator=g, device="cuda").float() for n in (M, N))
    bias = torch.randint(-8, 9, (N,), generator=g, device="cuda").float() / 4
    z = (a.double() @ w.double().t()) * sa.double()[:, None] * sw.double() + bias.double()
    for m in (None, M, max(M - 3, 0)):
        y = torch.full((M, N), 7.0, dtype=torch.float32 if wide else torch.bfloat16, device="cuda")
        fdl.fd_int_linear(a, sa, w, sw, y, bias=bias, gelu=gelu, m=None if m is None else count(m))
        n = M if m is None else m
        want = z[:n]
        if not gelu:
            assert torch.equal(y[:n], want.to(y.dtype))
        else:
            # (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)): the sum with tanh is known to 2^-53 only where it is exp(2 u), which at
            # z = -7 (6e-16) is 1 percent of it and below -8 all of it
            u = (2 / torch.pi) ** 0.5 * (want + 0.044715 * want ** 3)
            want = want / (1 + torch.exp(-2 * u))
            # beside the bound of gelu_err: from exp(-2 u) = 2^126 on (z = -10.1) the reciprocal is below the smallest normal
            # value, 2^-126, and may come as zero, so z times it is off by up to |z| 2^-126
            err = want.abs() * ((2 * 1.4426950408889634 * u).abs() * 2.0 ** -22 + 2.0 ** -21) + z[:n].abs().clamp(min=1) * 2.0 ** -126
            assert bool(((y[:n].double() - want).abs() <= err + UB * (want.abs() + err)).all())
        assert bool((y[n:] == 7).all())


def test_row_count_on_the_device_picks_the_tiles():
    """A capacity at which both tile kernels are launched: for every row count the bits of the call with just those rows."""
    N, K, cap = 1536, 6144, 9828
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    a, w = (torch.randint(-127, 128, (n, K), generator=g, device="cuda", dtype=torch.int32).to(torch.int8) for n in (cap, N))
    sa, sw = torch.rand(cap, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    for m in (9828, 5000, 300, 1, 0):
        gh.say(f"capacity {cap}, {m} rows")
        y, y2 = torch.full((cap, N), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty((max(m, 1), N), dtype=torch.bfloat16, device="cuda")
        fdl.fd_int_linear(a, sa, w, sw, y, m=count(m))
        if m:
            fdl.fd_int_linear(a[:m], sa[:m], w, sw, y2)
            assert torch.equal(y[:m], y2)       # the sums are exact, whatever the tile
        assert bool((y[m:] == 7).all())


@pytest.mark.parametrize("to", ["bf16", "codes", "ints"])
@pytest.mark.parametrize("rows,D,B,m", [(9001, 64, 40, 8999), (5001, 192, 9, 5001), (9001, 320, 40, 8999), (4099, 1024, 9, 4099), (3200, 1536, 2, 3200),
                                        (1500, 2064, 7, 1500), (1300, 4112, 4, 1290), (1100, 8208, 3, 1030)])
def test_norm_runs(rows, D, B, m, to):
    """Runs of several rows a team of 16 lanes to eight waves, whose requests begin inside a run, some of them empty: the bits of
    the same rows in calls of one request each."""
    gh.say(f"norm runs {rows}x{D} B={B} m={m} to={to}")
    rng = np.random.default_rng([rows, D])
    h, y = dev(rng.standard_normal((rows, D)).astype(np.float32)), bf16(rng.standard_normal((rows, D))).cuda()
    mod = dev((0.3 * rng.standard_normal((B, 3 * D))).astype(np.float32))
    cu = np.concatenate([[0], np.sort(rng.integers(0, m + 1, B - 1)), [m]]).astype(np.int32)
    if B > 2:
        cu[2] = cu[1]
    post, weight = (dev((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)) for _ in range(2))

    def run(x, yy, cu_q, n, mo):
        n_rows = x.shape[0]
        a = torch.full((n_rows, D), 7, dtype={"bf16": torch.bfloat16, "codes": torch.uint8, "ints": torch.int8}[to], device="cuda")
        s = {"bf16": None, "codes": torch.zeros((n_rows, scaled.stride(D)), dtype=torch.uint8, device="cuda"), "ints": torch.full((n_rows,), 7.0, device="cuda")}[to]
        fdl.fd_norm_residual(x, a, cu_q, count(n), y=yy, post_weight=post, gate=mo[:, 2 * D:], residual=0.5, weight=weight, shift=mo[:, :D],
                             mod_scale=mo[:, D:2 * D], a_scale=s)
        return x, a, s

    x, a, s = run(h.clone(), y, dev(cu), m, mod)
    for b in range(B):
        r = slice(int(cu[b]), int(cu[b + 1]))
        if r.start == r.stop:
            continue
        x2, a2, s2 = run(h[r].clone(), y[r].contiguous(), None, r.stop - r.start, mod[b:b + 1])
        assert torch.equal(x[r], x2) and torch.equal(a[r], a2) and (s is None or torch.equal(s[r], s2))
    assert torch.equal(x[m:], h[m:]) and bool((a[m:] == 7).all())
