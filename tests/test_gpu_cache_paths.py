"""The attention over an 8-bit cache where its kernel takes another path: more items than workgroups, whole and cut, of one length
and mixed; many requests; both ways by the row count on the device; a capacity above the rows; other streams and recorded calls."""
import numpy as np
import pytest
import torch

from oracle import integer as ref
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_cache import cache, check_attention, run_attention
from tests.test_gpu_scaled import bf16, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


def offsets(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def make(q_len, k_len, hq, hk, dh, extra=0, seed=0):
    rng = np.random.default_rng([seed, dh, hq, sum(q_len)])
    tokens, rows = sum(k_len), sum(q_len) + extra
    k, ks = cache(rng, tokens, hk, dh)
    v, vs = cache(rng, tokens, hk, dh)
    q = bf16(rng.standard_normal((rows, hq * dh)) * np.exp(0.5 * rng.standard_normal((rows, 1))))
    return (q, k, ks, v, vs, offsets(q_len), offsets(k_len), hq, hk, dh)


# (queries, keys, heads, key heads, head dim): items in whole rounds; more items than workgroups, mixed lengths (cut); one long item a
# head, cut into many pieces; 65 and 200 requests (tables by threads); few rows of many requests; a request of more rows than a
# tile beside requests of one
SHAPES = {
    "whole": ([2100], [600], 24, 24, 64),
    "mixed": ([40, 900, 300, 1, 700], [200, 2600, 64, 3000, 1100], 24, 8, 64),
    "mixed128": ([500, 0, 250, 900], [1500, 77, 2100, 300], 16, 16, 128),
    "pieces": ([300], [9000], 2, 2, 128),
    "pieces64": ([200], [12000], 3, 1, 64),
    "few": ([90], [9000], 2, 2, 128),
    "few16": ([30], [5000], 6, 2, 16),
    "requests65": ([3] * 65, [50 + i for i in range(65)], 2, 2, 64),
    "requests200": ([1 + 37 * (i % 5) for i in range(200)], [1 + (i * 53) % 400 for i in range(200)], 4, 2, 64),
    "requests200few": ([i % 3 for i in range(200)], [(i * 53) % 400 for i in range(200)], 4, 4, 128),
    "beside": ([1, 700, 1, 1], [900, 900, 3, 2000], 4, 2, 16),
}


@pytest.mark.parametrize("name", list(SHAPES))
def test_attention_paths(name):
    gh.say(f"cache attention {name}: {SHAPES[name][2:]}")
    case = make(*SHAPES[name])
    got = run_attention(*case, longest=max(SHAPES[name][1]))
    check_attention(got, *case)


def test_one_thousand_requests():
    """The most requests of a call, half of them without rows or tokens, of both ways' lengths."""
    rng = np.random.default_rng(4)
    q_len, k_len = rng.integers(0, 5, 1024) * (rng.random(1024) < 0.6), rng.integers(0, 90, 1024)
    case = make(q_len.tolist(), k_len.tolist(), 2, 1, 64)
    check_attention(run_attention(*case, longest=89), *case)
    q_len[500] = 2000                                        # and in tiles
    case = make(q_len.tolist(), k_len.tolist(), 2, 1, 64)
    check_attention(run_attention(*case, longest=89), *case)


@pytest.mark.parametrize("rows", [1, 33, 96, 97, 129, 257])
def test_capacity_above_the_rows(rows):
    """A step passes the capacity of all tokens: the way is picked on the device, and the results are within the bound there too;
    the longest request may be named too long."""
    case = make([rows, 0], [3000, 10], 4, 4, 128, extra=700)
    got = run_attention(*case)
    check_attention(got, *case)
    tight = (case[0][:rows].contiguous(), *case[1:])
    check_attention(run_attention(*tight, longest=3000), *tight)


def test_longest_request_named_too_short():
    """max_request_tokens sizes the launch; a request that is longer is run all the same, uncut."""
    case = make([5, 300], [3000, 2000], 2, 2, 64)
    check_attention(run_attention(*case, longest=10), *case)


def test_other_stream():
    """On a stream of its own, after work there; and two calls at once on two streams, each with its workspace."""
    cases = [make([300], [4000], 4, 4, 64, seed=1), make([20], [6000], 4, 4, 64, seed=2)]
    want = [run_attention(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    done = []
    for c, s in zip(cases, streams):
        q, k, ks, v, vs, cu, off, hq, hk, dh = c
        with torch.cuda.stream(s):
            t = [torch.empty_like(x) for x in (q.cuda(), dev(k), dev(ks), dev(v), dev(vs), dev(cu), dev(off))]
            for a, b in zip(t, (q.cuda(), dev(k), dev(ks), dev(v), dev(vs), dev(cu), dev(off))):
                a.copy_(b)
            o = torch.empty((q.shape[0], hq * dh), dtype=torch.bfloat16, device="cuda")
            ws = torch.empty(fdl.fd_cache_attention_ws_size(q.shape[0], hq, hk, dh), dtype=torch.uint8, device="cuda")
        done.append((t, o, ws, s, c))
    torch.cuda.synchronize()
    for _ in range(3):
        for t, o, ws, s, c in done:
            fdl.fd_cache_attention(t[0], t[1], t[2], t[3], t[4], o, t[5], t[6], *c[7:], ws, stream=s)
    torch.cuda.synchronize()
    for (_, o, _, _, c), w in zip(done, want):
        np.testing.assert_array_equal(o.double().cpu().numpy().reshape(w.shape), w)


def test_recorded():
    """Recorded once and replayed on changing queries and offsets (few rows, then tiles, then none), with eager work between."""
    hq, hk, dh, rows, tokens = 4, 2, 128, 400, 5000
    rng = np.random.default_rng(9)
    k, ks = cache(rng, tokens, hk, dh)
    v, vs = cache(rng, tokens, hk, dh)
    d = [dev(x) for x in (k, ks, v, vs)]
    q = torch.zeros((rows, hq * dh), dtype=torch.bfloat16, device="cuda")
    cu, off = torch.zeros(3, dtype=torch.int32, device="cuda"), dev(np.array([0, 4000, 5000], np.int32))
    o = torch.zeros_like(q)
    ws = torch.empty(fdl.fd_cache_attention_ws_size(rows, hq, hk, dh), dtype=torch.uint8, device="cuda")
    call = lambda: fdl.fd_cache_attention(q, d[0], d[1], d[2], d[3], o, cu, off, hq, hk, dh, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for q_len in ([3, 2], [200, 200], [0, 0], [1, 0], [0, 400], [3, 2]):
        q.copy_(bf16(rng.standard_normal((rows, hq * dh))))
        cu.copy_(dev(offsets(q_len)))
        o.fill_(7)
        call()
        torch.cuda.synchronize()
        eager = o.clone()
        _ = (torch.randn(1 << 14, device="cuda") * 2).sum().item()
        o.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, eager)
        case = (q.cpu(), k, ks, v, vs, offsets(q_len), np.array([0, 4000, 5000], np.int32), hq, hk, dh)
        check_attention(o.double().cpu().numpy().reshape(rows, hq, dh), *case)


@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("dh", [16, 64, 128])
def test_pieces_of_keys_without_weight(rows, dh):
    """Scores of the first half of the keys below the lowest fp32 value: those keys have the weight zero, also where a piece of the cut range has
    no others, and the result is that of the second half."""
    rng = np.random.default_rng([rows, dh])
    tokens, half, hk = 6000, 3000, 2
    x = rng.standard_normal((tokens, hk, dh))
    x[:half, :, 0], x[half:, :, 0] = 448.0, 0.0
    (k, ks), (v, vs) = ref.head_codes(x), ref.head_codes(rng.standard_normal((tokens, hk, dh)))
    q = bf16(rng.standard_normal((rows, hk * dh)))
    k, v, ks, vs = k.reshape(tokens, -1), v.reshape(tokens, -1), ks.T.copy(), vs.T.copy()
    q[:, ::dh] = -2e38                       # times 448: past fp32's range
    got = run_attention(q, k, ks, v, vs, offsets([rows]), offsets([tokens]), hk, hk, dh)
    q[:, ::dh] = 0                           # the second half's values there are zeros
    check_attention(got, q, k[half:], ks[:, half:].copy(), v[half:], vs[:, half:].copy(), offsets([rows]), offsets([half]), hk, hk, dh)
