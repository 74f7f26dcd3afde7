"""The 8-bit block (fd_scaled_block_forward) and the step that runs it: against the 64-bit reference, against its own
operators one by one, through SparseStep eager and recorded, and as the source of the importance signal."""
import numpy as np
import pytest
import torch

from oracle import scaled as ref
from paper_2607_12121_amd import flashdiff as fdl
from paper_2607_12121_amd import workloads as wl
from tests import gpu_harness as gh
from tests.helpers import rel_err, small_workload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


WORK = {
    "tiny": lambda: wl.WORKLOADS["tiny"],
    # two requests of different grids, hidden 1088 (a last block of half a block), head dim 64
    "odd": lambda: small_workload("image", requests=(wl.RequestShape("grid2d", (9, 13), (4, 4)), wl.RequestShape("grid2d", (16, 20), (4, 5))),
                                  activity="frac", activity_args=(0.3, 0.6), L=2, D=1088, H=17, dh=64, F=2112),
    # a short video, head dim 128
    "video": lambda: small_workload("video", requests=(wl.RequestShape("grid3d", (4, 10, 12), (2, 5, 4)),), activity="count", activity_args=(5,),
                                    L=1, D=256, H=2, dh=128, F=1024),
    # every row of 30 requests (most of one or two tokens), more rows than the few-row kernels take
    "many": lambda: small_workload("audio", requests=tuple(wl.RequestShape("seq", (1 + (n % 7) * 5,), (8,)) for n in range(30)),
                                   activity="frac", activity_args=(1.0, 1.0), L=1, D=128, H=8, dh=16, F=384),
}
ROPE = {16: dict(dims=[8, 8], theta=[1e4, 1e4], step=[1.0, 1.0], halves=True), 64: dict(dims=[24, 40], theta=[1e4, 100.0], step=[1.0, 0.5], halves=False),
        128: dict(dims=[44, 42, 42], theta=[1e4] * 3, step=[1.0] * 3, halves=False)}


def coords(w, axes):
    """Token positions: each request's grid, leading axes 0 where it has fewer than `axes`."""
    out = []
    for rq in w.requests:
        c = np.indices(rq.dims).reshape(len(rq.dims), -1).T[:, -axes:]
        out.append(np.concatenate([np.zeros((len(c), axes - c.shape[1]), np.int64), c], 1))
    return np.concatenate(out).astype(np.int32)


def make(name, with_rope=True):
    w = WORK[name]()
    case = gh.make_case(w.name, workload=w)
    rng = np.random.default_rng(w.N)
    params = dict(case.params_gpu)
    for k in ("norm_1", "norm_2"):
        params[k] = torch.from_numpy((1 + 0.1 * rng.standard_normal((w.L, w.D))).astype(np.float32)).cuda()
    scaled = fdl.scaled_params(params)
    rope = dict(ROPE[w.dh]) if with_rope else None
    pos = coords(w, len(rope["dims"])) if rope else None
    return case, scaled, rope, pos


def step_of(case, scaled, rope, pos):
    return fdl.SparseStep(case.plan, case.dims, case.params_gpu, case.w.L, k_cache=case.k_cache.cuda(), v_cache=case.v_cache.cuda(),
                          scaled=scaled, rope=fdl.rope_axes(**rope) if rope else None, coord=torch.from_numpy(pos).cuda() if rope else None)


def run_step(case, st, **kw):
    x, xp = torch.from_numpy(case.inp.x_cur).cuda(), torch.from_numpy(case.inp.x_prev).cuda()
    st.step(x, xp, torch.from_numpy(case.inp.eps).cuda(), torch.from_numpy(wl.dt_per_request(case.w)).cuda(), case.cond.cuda(), **kw)
    torch.cuda.synchronize()
    return x


@pytest.mark.parametrize("with_rope", [True, False])
@pytest.mark.parametrize("name", list(WORK))
def test_step_is_its_operators(name, with_rope):
    """A step's blocks are, bit for bit, their operators called one by one (each held to its 64-bit reference in
    test_gpu_scaled.py) around the attention, whose output is taken from the block's workspace and held to
    softmax(q k^T) v of the bf16 operands in 64 bits; rows of skipped tokens stay.  (A 64-bit chain beside it would show
    less: codes round by 2^-4, and a value next to a limit that one side rounds up and the other down differs by a whole
    step.)"""
    case, scaled, rope, pos = make(name, with_rope)
    w, d = case.w, case.dims
    gh.say(f"8-bit step {name}: N={w.N} D={w.D} F={w.F} L={w.L} rope={rope}")
    st = step_of(case, scaled, rope, pos)
    run_step(case, st)
    N, D, F = w.N, w.D, w.F
    M = int(st.m.item())
    idx = st.idx[:M].long()
    assert M > 0
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    at = up(w.B * 6 * D * 4) + 2 * up(N * D * 2)           # modulation, norm's rows, queries, then the attention's output
    code = lambda n: (torch.empty((N, n), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((N, fdl.fd_scale_stride(n)), dtype=torch.uint8, device="cuda"))  # noqa: E731
    rows16 = lambda n: torch.empty((N, n), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    num = lambda t: t.double().cpu().numpy().reshape(-1, w.H, w.dh)  # noqa: E731
    cu, off = st.cu_q.cpu().numpy(), case.rmap.req_tok_off
    h, h2 = torch.zeros((N, D), device="cuda"), torch.zeros((N, D), device="cuda")
    for t in (h, h2):
        fdl.fd_embed(case.plan, d, st.xa, case.params_gpu["w_e"], case.params_gpu["b_e"], case.params_gpu["pos"], st.idx, st.m, t)
    (a, sa), (g, sg), qkv, q, y = code(D), code(F), rows16(3 * D), rows16(D), rows16(D)
    for l in range(w.L):
        p = {k: t[l] for k, t in scaled.items() if t.dim() > 1 and t.shape[0] == w.L and k != "pos"}
        mod = st.mod[l]
        part = lambda i: mod[:, i * D:(i + 1) * D]  # noqa: E731
        k1, v1 = case.k_cache[l].cuda(), case.v_cache[l].cuda()
        k2, v2 = k1.clone(), v1.clone()
        fdl.fd_scaled_block_forward(case.plan, d, st.block_w[l], st.rope, st.coord, h, st.idx, st.cu_q, st.m, k1, v1, st.ws_block)
        o = st.ws_block[at:at + N * D * 2].view(torch.bfloat16).view(N, D).clone()

        fdl.fd_rms_quant(h2, a, sa, st.cu_q, st.m, weight=p["norm_1"], shift=part(0), mod_scale=part(1))
        fdl.fd_scaled_linear(a, sa, p["w_qkv"], p["s_qkv"], qkv, bias=p["b_qkv"], m=st.m)
        if rope:
            fdl.fd_rope_axes(qkv, st.coord, st.idx, st.m, q, k2, v2, heads=w.H, kv_heads=w.H, head_dim=w.dh, rope=st.rope)
        else:
            q[:M], k2[idx], v2[idx] = qkv[:M, :D], qkv[:M, D:2 * D], qkv[:M, 2 * D:]
        assert torch.equal(k1, k2) and torch.equal(v1, v2), l
        assert torch.equal(k1, st.k_cache[l]) and torch.equal(v1, st.v_cache[l]), l
        fdl.fd_quant_blocks(o, 1, a, sa, m=st.m)
        fdl.fd_scaled_linear(a, sa, p["w_o"], p["s_o"], y, bias=p["b_o"], m=st.m)
        fdl.fd_rms_quant(h2, a, sa, st.cu_q, st.m, y=y, gate=part(2), weight=p["norm_2"], shift=part(3), mod_scale=part(4))
        fdl.fd_scaled_linear(a, sa, p["w_1"], p["s_1"], g, sg, bias=p["b_1"], gelu=True, m=st.m)
        fdl.fd_scaled_linear(g, sg, p["w_2"], p["s_2"], y, bias=p["b_2"], m=st.m)
        fdl.fd_rms_quant(h2, None, None, st.cu_q, st.m, y=y, gate=part(5))
        assert torch.equal(h, h2), l
        q64, k64, v64, o64 = num(q[:M]), num(k1), num(v1), num(o[:M])
        for b in range(w.B):
            if cu[b] == cu[b + 1]:
                continue
            s = np.einsum("mhd,nhd->hmn", q64[cu[b]:cu[b + 1]], k64[off[b]:off[b + 1]]) / np.sqrt(w.dh)
            e = np.exp(s - s.max(-1, keepdims=True))
            want = np.einsum("hmn,nhd->mhd", e / e.sum(-1, keepdims=True), v64[off[b]:off[b + 1]])
            assert rel_err(o64[cu[b]:cu[b + 1]], want) <= gh.TOL, (l, b)
        skipped = np.setdiff1d(np.arange(N), idx.cpu().numpy())
        assert torch.equal(k1.cpu()[skipped], case.k_cache[l][skipped]) and torch.equal(v1.cpu()[skipped], case.v_cache[l][skipped])
    assert torch.equal(h[:M], st.h[:M]) and bool((h[M:] == 0).all())
    assert not torch.isnan(h[:M]).any() and not torch.equal(h[:M], torch.zeros_like(h[:M]))


def test_no_active_rows():
    """A threshold of infinity: no row is active, and latent, caches and hidden rows stay."""
    case, scaled, rope, pos = make("odd")
    st = step_of(case, scaled, rope, pos)
    st.h.fill_(3.0)
    x = torch.from_numpy(case.inp.x_cur).cuda()
    st.step(x, torch.from_numpy(case.inp.x_prev).cuda(), torch.full((case.w.B,), float("inf"), dtype=torch.float64, device="cuda"),
            torch.from_numpy(wl.dt_per_request(case.w)).cuda(), case.cond.cuda())
    torch.cuda.synchronize()
    assert int(st.m.item()) == 0
    assert np.array_equal(x.cpu().numpy(), case.inp.x_cur) and bool((st.h == 3.0).all())
    assert torch.equal(st.k_cache.cpu(), case.k_cache) and torch.equal(st.v_cache.cpu(), case.v_cache)


def test_step_recorded():
    """One step recorded and replayed on changing latents, with eager work between: the eager step's bits."""
    case, scaled, rope, pos = make("odd")
    w = case.w
    eager, rec = step_of(case, scaled, rope, pos), step_of(case, scaled, rope, pos)
    dt, cond = torch.from_numpy(wl.dt_per_request(w)).cuda(), case.cond.cuda()
    xg, xpg, eg = torch.empty((w.N, w.C), device="cuda"), torch.empty((w.N, w.C), device="cuda"), torch.empty(w.B, dtype=torch.float64, device="cuda")
    graph = rec.capture(xg, xpg, eg, dt, cond, max_skip=2)
    for n in range(3):
        inp = wl.step_inputs(w, n, rmap=case.rmap)
        x, xp, eps = torch.from_numpy(inp.x_cur).cuda(), torch.from_numpy(inp.x_prev).cuda(), torch.from_numpy(inp.eps).cuda()
        xg.copy_(x); xpg.copy_(xp); eg.copy_(eps)
        eager.step(x, xp, eps, dt, cond, max_skip=2)
        torch.cuda.synchronize()
        _ = (torch.randn(1 << 14, device="cuda") * 2).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        M = int(eager.m.item())
        for a, b, what in ((xg, x, "latent"), (rec.h[:M], eager.h[:M], "h"), (rec.v[:M], eager.v[:M], "v"), (rec.k_cache, eager.k_cache, "K"),
                           (rec.v_cache, eager.v_cache, "V")):
            assert torch.equal(a, b), f"replay {n}: {what}"


def test_importance_after_the_block():
    """fd_region_importance on the 8-bit block's workspace: the block's own queries (from its operators) against its
    keys, in 64 bits; bf16 queries and keys enter both, so the tolerance is the importance tests' own, 2e-2."""
    case, scaled, rope, pos = make("tiny")
    w = case.w
    st = step_of(case, scaled, rope, pos)
    run_step(case, st, importance_block=0)
    M, D = int(st.m.item()), w.D
    idx = st.idx[:M].cpu().numpy()
    h = torch.empty((w.N, D), device="cuda")
    fdl.fd_embed(case.plan, case.dims, st.xa, case.params_gpu["w_e"], case.params_gpu["b_e"], case.params_gpu["pos"], st.idx, st.m, h)
    q = torch.empty((w.N, D), dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty((w.N, fdl.fd_scale_stride(D)), dtype=torch.uint8, device="cuda")
    mod = st.mod[0]
    fdl.fd_rms_quant(h, q, s, st.cu_q, st.m, weight=scaled["norm_1"][0], shift=mod[:, :D], mod_scale=mod[:, D:2 * D])
    qkv = torch.empty((w.N, 3 * D), dtype=torch.bfloat16, device="cuda")
    fdl.fd_scaled_linear(q, s, scaled["w_qkv"][0], scaled["s_qkv"][0], qkv, bias=scaled["b_qkv"][0], m=st.m)
    rq, k, v = (torch.empty((w.N, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    fdl.fd_rope_axes(qkv, st.coord, st.idx, st.m, rq, k, v, heads=w.H, kv_heads=w.H, head_dim=w.dh, rope=st.rope)
    q64 = rq[:M].double().cpu().numpy().reshape(M, w.H, w.dh)
    k64 = st.k_cache[0].double().cpu().numpy().reshape(w.N, w.H, w.dh)
    reg = case.rmap.token_region
    logits = np.einsum("mhd,nhd->hmn", q64, k64) / np.sqrt(w.dh)
    p = np.exp(logits - logits.max(-1, keepdims=True))
    p = (p / p.sum(-1, keepdims=True)).mean(0)
    got = st.importance.cpu().numpy()
    active = st.active.cpu().numpy().astype(bool)
    for r in np.nonzero(active)[0]:
        rows, toks = np.nonzero(reg[idx] == r)[0], np.nonzero(reg == r)[0]
        want = p[np.ix_(rows, toks)].sum() / len(toks) ** 2
        assert abs(got[r] - want) <= gh.TOL * want
    assert np.all(np.isnan(got[~active]))


def test_refusals():
    case, scaled, rope, pos = make("tiny")
    st = step_of(case, scaled, rope, pos)
    args = (st.h, st.idx, st.cu_q, st.m, st.k_cache[0], st.v_cache[0])
    f = fdl.fd_scaled_block_forward
    for call in (lambda: f(case.plan, case.dims, st.block_w[0], st.rope, None, *args, st.ws_block),
                 lambda: f(case.plan, case.dims, st.block_w[0], st.rope, st.coord[:, :1].contiguous(), *args, st.ws_block),
                 lambda: f(case.plan, case.dims, st.block_w[0], st.rope, st.coord, *args, st.ws_block[:-256]),
                 lambda: f(case.plan, case.dims, fdl.FdScaledWeights(), st.rope, st.coord, *args, st.ws_block),
                 lambda: f(case.plan, case.dims, st.block_w[0], fdl.rope_axes([10, 10]), st.coord, *args, st.ws_block),
                 lambda: fdl.SparseStep(case.plan, case.dims, case.params_gpu, 1, rope=st.rope, coord=st.coord)):
        with pytest.raises(fdl.FlashDiffError):
            call()
