"""Attention over the 8-bit cache against the same formula in 64 bits on the values that the cache stands for.

Tolerances, from the roundings (u16 = half a step of the output's type: 2^-11 fp16, 2^-8 bf16):
  score   the products are exact in fp32 (fp16 x 8-bit), their sum over D channels is off by at most D 2^-24 sum|q k|; two more
          roundings, and the softmax scale's, each 2^-24 of the score itself (which sum|q k| bounds).  With e = scale (D + 8) 2^-24
          max_t sum|q_c k_c| the relative error of a weight p is 2 e + 2^-20 (its own score, the row's sum; exponential and sums).
  out     |o - o'| <= (2^-11 + 2 e + 2^-19) (sum p|v| + |o|) + 2^-24 sum_t |v_t| + u16 |o|: weights rounded to fp16 (2^-11 relative,
          2^-25 absolute where they are subnormal next to the row's largest weight) and divided by their own sum: with relative errors
          d_t, o' - o = sum p d_t (v_t - o) / (1 + sum p d_t), and |v_t - o| <= |v_t| + |o|; then the output's rounding
  lse     e + 2^-21 (1 + |lse|)
  weights sum of p (2 e + 2^-20) over the rows + 2^-23 |the result|
"""
import numpy as np
import pytest

from tests import q8_reference as R
from tests.test_gpu_q8_cache import Device, append, dtypes

pytestmark = pytest.mark.gpu
INT8, E4M3 = R.INT8, R.E4M3


def make(api, seed, code, D, io, hkv, ratio, lens, max_len, page=0, drop=(), spread=0.5):
    rng = np.random.default_rng(seed)
    dev = Device(api, rng, code, D, hkv, len(lens), max_len, page, dtypes()[io], ratio, drop)
    if max(lens) > 0:
        append(dev, rng, [0] * len(lens), lens, max(lens), spread=spread)
    return rng, dev


def queries(rng, dev, ratio, n_q, spread=1.0, strided=False):
    import torch
    hq = dev.hkv * ratio
    x = rng.standard_normal((dev.batch, n_q, hq, dev.D)) * np.exp(spread * rng.standard_normal((dev.batch, n_q, hq, 1)))
    q = torch.from_numpy(x).to(dev.shape.dtype)
    ref = q.double().numpy()
    q = q.cuda()
    if strided:   # by heads first, wider rows
        wide = torch.full((dev.batch, hq, n_q, dev.D + 24), float("nan"), dtype=q.dtype, device="cuda")
        wide[..., :dev.D] = q.transpose(1, 2)
        q = wide[..., :dev.D].transpose(1, 2)
    return q, ref


def compare(dev, ref_q, out, lse, lens, nq, scale, causal, ratio, out0, lse0, weights=None, w_in=None, w0=None):
    D, u16 = dev.D, {"torch.float16": 2.0 ** -11, "torch.bfloat16": 2.0 ** -8}[str(dev.shape.dtype)]
    n_q = ref_q.shape[1]
    for b in range(dev.batch):
        n, m = lens[b], nq[b]
        assert np.array_equal(out[b, m:], out0[b, m:]) and np.array_equal(lse[b, m:], lse0[b, m:])   # rows behind the last query
        i = np.arange(m)
        for h in range(dev.hkv):
            k, v = dev.ref["k"][b][h].rows(n), dev.ref["v"][b][h].rows(n)
            exists = np.array([dev.pages("k", b, t // 64) is not None and dev.pages("v", b, t // 64) is not None for t in range(n)], dtype=bool)
            total, slack = np.zeros(n), np.zeros(n)
            for g in range(ratio):
                hq = h * ratio + g
                q = ref_q[b, :m, hq]
                vis = np.clip(n - m + 1 + i, 0, n) if causal else np.full(m, n)
                seen = (np.arange(n)[None, :] < vis[:, None]) & exists[None, :]
                o, z, p, pv = R.attention(q, k, v, scale, seen)
                e = abs(scale) * (D + 8) * 2.0 ** -24 * np.where(seen, np.abs(q) @ np.abs(k).T, 0).max(axis=1, initial=0.0)
                tol = (2.0 ** -11 + 2 * e[:, None] + 2.0 ** -19) * (pv + np.abs(o)) + 2.0 ** -24 * (seen @ np.abs(v)) + u16 * np.abs(o)
                tol = tol * (1 + u16) + 2.0 ** -25      # (the output's rounding of what is already off; its subnormal step)
                d = np.abs(out[b, :m, hq] - o)
                assert (d <= tol).all(), (b, h, g, float((d / tol).max()))
                none = ~seen.any(axis=1)
                assert (out[b, :m, hq][none] == 0).all() and (lse[b, :m, hq][none] == -np.inf).all()
                dz = np.abs(lse[b, :m, hq][~none] - z[~none])
                assert (dz <= e[~none] + 2.0 ** -21 * (1 + np.abs(z[~none]))).all(), float(dz.max())
                total += p.sum(axis=0)
                slack += (p * (2 * e[:, None] + 2.0 ** -20)).sum(axis=0)
            if weights is not None:
                ref = total + (0 if w_in is None else w_in[b, h, :n])
                d = np.abs(weights[b, h, :n] - ref)
                assert (d <= slack + 2.0 ** -23 * np.abs(ref) + 2.0 ** -126).all(), (b, h, float((d - slack).max()))
                assert np.array_equal(weights[b, h, n:], w0[b, h, n:])


def run(api, rng, dev, ratio, lens, n_q, nq=None, causal=False, weights=False, splits=0, strided=False, in_place=False, bound=None,
        spread=1.0, no_weights_in=False):
    import torch
    q, ref_q = queries(rng, dev, ratio, n_q, spread, strided)
    B, hq, D = dev.batch, dev.hkv * ratio, dev.D
    scale = 1.0 / np.sqrt(D)
    out = torch.full((B, n_q, hq, D), 5.0, dtype=dev.shape.dtype, device="cuda")
    lse = torch.full((B, n_q, hq), 5.0, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    w_in = w_out = w0 = w_ref = None
    if weights:
        w_in = torch.from_numpy(rng.random((B, dev.hkv, dev.max_len)).astype(np.float32)).cuda()
        w_ref = w_in.double().cpu().numpy()
        w_out = w_in if in_place else torch.full_like(w_in, 9.0)
        w0 = w_out.cpu().numpy()
        if no_weights_in:
            w_in = w_ref = None
    api.nsn_q8_attention(dev.shape, q, dev.cache["k"], dev.cache["v"], i32(lens), max(lens) if bound is None else bound, scale, causal=causal,
                         q_lens=None if nq is None else i32(nq), weights_in=w_in, weights_out=w_out, n_splits=splits, out=out, lse=lse)
    torch.cuda.synchronize()
    nq = [n_q] * B if nq is None else nq
    nq = [min(max(x, 0), n_q) for x in nq]
    compare(dev, ref_q, out.double().cpu().numpy(), lse.cpu().numpy(), lens, nq, scale, causal, ratio,
            np.full((B, n_q, hq, D), 5.0), np.full((B, n_q, hq), 5.0, np.float32), None if w_out is None else w_out.cpu().numpy(), w_ref, w0)


@pytest.mark.parametrize("io", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("code", [INT8, E4M3])
@pytest.mark.parametrize("page", [0, 64, 192])
def test_single_tokens(gpu_api, code, D, io, page):
    """Lengths of zero, one, and around the blocks."""
    lens = [0, 1, 63, 64, 65, 500, 576]
    rng, dev = make(gpu_api, 1 + D + page, code, D, io, 2, 4, lens, 576, page)
    for splits in (0, 1, 2, 9):
        run(gpu_api, rng, dev, 4, lens, 1, splits=splits, strided=splits == 2, weights=splits != 1, in_place=splits == 9)
    run(gpu_api, rng, dev, 4, lens, 1, bound=576, weights=True, no_weights_in=True)


@pytest.mark.parametrize("ratio", [1, 2, 3, 5, 7, 8, 16, 17, 33])
def test_head_layouts(gpu_api, ratio):
    lens = [130, 67]
    for code, io, D in ((INT8, "fp16", 128), (E4M3, "bf16", 64)):
        rng, dev = make(gpu_api, 50 + ratio, code, D, io, 3, ratio, lens, 192)
        run(gpu_api, rng, dev, ratio, lens, 1, weights=True)
        run(gpu_api, rng, dev, ratio, lens, 3, causal=True, weights=True, splits=2)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("code,D,io", [(INT8, 128, "fp16"), (INT8, 64, "bf16"), (E4M3, 128, "bf16"), (E4M3, 64, "fp16")])
@pytest.mark.parametrize("n_q,ratio", [(2, 1), (5, 4), (16, 1), (17, 2), (33, 1), (40, 4), (129, 1), (70, 3), (300, 2)])
def test_chunks(gpu_api, code, D, io, n_q, ratio, causal):
    """Chunks longer and shorter than the cache (rows that see nothing), ragged and empty ones."""
    lens = [0, 1, 64, 130, 300, 448]
    rng, dev = make(gpu_api, n_q + D, code, D, io, 2, ratio, lens, 448, 64 if n_q % 2 else 0)
    run(gpu_api, rng, dev, ratio, lens, n_q, causal=causal, weights=True)
    nq = [n_q, 0, n_q - 1, 1, n_q + 5, max(1, n_q // 2)]
    run(gpu_api, rng, dev, ratio, lens, n_q, nq=nq, causal=causal, weights=n_q % 2 == 1, strided=True, splits=0 if ratio == 1 else 3)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("code,D,io,page", [(INT8, 128, "fp16", 0), (INT8, 64, "bf16", 128), (E4M3, 128, "bf16", 64), (E4M3, 64, "fp16", 0)])
@pytest.mark.parametrize("n_q,ratio", [(33, 1), (20, 3), (129, 1), (70, 4)])
def test_chunks_of_many_heads(gpu_api, code, D, io, page, n_q, ratio, causal):
    """Enough units that rows go 128 at a time: whole and ragged chunks, longer and shorter than the cache, empty ones, cut into runs."""
    lens = [0, 1, 64, 130, 384, 300, 65, 256]
    rng, dev = make(gpu_api, n_q + D, code, D, io, 16, ratio, lens, 384, page)
    run(gpu_api, rng, dev, ratio, lens, n_q, causal=causal, weights=n_q == 20, strided=n_q == 70)
    nq = [n_q, 0, n_q - 1, 1, n_q + 5, n_q // 2, n_q, 7]
    run(gpu_api, rng, dev, ratio, lens, n_q, nq=nq, causal=causal, weights=n_q == 33, splits=3 if n_q > 100 else 0)


@pytest.mark.parametrize("code,D", [(INT8, 128), (E4M3, 64)])
def test_a_long_chunk_of_few_heads(gpu_api, code, D):
    """So much work that rows go 128 at a time although there are few units: each reaches into many runs."""
    lens = [14001]
    rng, dev = make(gpu_api, 3 + D, code, D, "bf16", 1, 1, lens, 14016)
    run(gpu_api, rng, dev, 1, lens, 2048, nq=[150], causal=True, weights=True)
    run(gpu_api, rng, dev, 1, lens, 2048, nq=[129])


@pytest.mark.parametrize("code,D,n_q,lens", [(INT8, 64, 260, [107000]), (E4M3, 128, 150, [60000, 30000, 40])])
def test_a_few_tiles_over_very_many_tokens(gpu_api, code, D, n_q, lens):
    """A tile of rows that reaches into far more than sixteen runs: its sums are joined in two steps."""
    rng, dev = make(gpu_api, 83, code, D, "bf16", 1, 1, lens, 107008 if D == 64 else 60032)
    run(gpu_api, rng, dev, 1, lens, n_q, causal=True, spread=0.3)
    run(gpu_api, rng, dev, 1, lens, n_q, splits=23, spread=0.3)


@pytest.mark.parametrize("code,D,io", [(INT8, 128, "fp16"), (E4M3, 64, "bf16")])
@pytest.mark.parametrize("n_q,ratio", [(1, 1), (1, 5), (3, 7)])
def test_units_that_reach_into_many_runs(gpu_api, code, D, io, n_q, ratio):
    """More than 64 runs to a unit: their partial sums are joined in two steps; and just so many."""
    lens = [6001, 4096, 4097, 70]
    rng, dev = make(gpu_api, 7 + D, code, D, io, 1, ratio, lens, 6016)
    for splits in (100, 40, 7):
        run(gpu_api, rng, dev, ratio, lens, n_q, splits=splits, causal=True, weights=splits == 100)


@pytest.mark.parametrize("n_q,causal", [(1, False), (9, True), (150, True), (150, False)])
@pytest.mark.parametrize("code", [INT8, E4M3])
def test_pages_that_do_not_exist_hold_no_tokens(gpu_api, code, n_q, causal):
    lens = [512, 300, 130]
    drop = [(0, 1, -1), (1, 0, 10 ** 9), (1, 2, 27), (2, 0, -7), (2, 1, -2 ** 31), (0, 3, 10)]
    rng, dev = make(gpu_api, 77, code, 128, "fp16", 2, 2, lens, 512, 128, drop=drop)
    for splits in (0, 1, 3):
        run(gpu_api, rng, dev, 2, lens, n_q, causal=causal, weights=True, splits=splits)


@pytest.mark.parametrize("n_q", [1, 40])
def test_lengths_outside_the_bounds_are_taken_as_within(gpu_api, n_q):
    import torch
    rng, dev = make(gpu_api, 5, INT8, 128, "fp16", 1, 2, [200, 200, 200], 256)
    q, ref = queries(rng, dev, 2, n_q)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    call = lambda lens, bound, nq: gpu_api.nsn_q8_attention(dev.shape, q, dev.cache["k"], dev.cache["v"], i32(lens), bound, 0.1,  # noqa: E731
                                                            q_lens=i32(nq))
    a, b = call([-3, 2 ** 31 - 1, 100], 150, [n_q + 9, n_q, -4]), call([0, 150, 100], 150, [n_q, n_q, 0])
    torch.cuda.synchronize()
    assert torch.equal(a, b) and not a[0].any() and not a[2].any() and a[1].any()


@pytest.mark.parametrize("n_q", [1, 64])
@pytest.mark.parametrize("io", ["fp16", "bf16"])
def test_large_and_small_scores_and_values(gpu_api, io, n_q):
    """Softmax rows that one token holds, and values over a wide range of scales."""
    import torch
    lens = [700, 90]
    for code in (INT8, E4M3):
        rng, dev = make(gpu_api, 9, code, 128, io, 1, 4, lens, 704, spread=1.5)
        run(gpu_api, rng, dev, 4, lens, n_q, weights=True, spread=1.2)
        run(gpu_api, rng, dev, 4, lens, n_q, weights=True, spread=0.0)


@pytest.mark.parametrize("n_q,hkv", [(1, 2), (40, 64)])
@pytest.mark.parametrize("code", [INT8, E4M3])
def test_scales_that_jump_from_block_to_block(gpu_api, code, n_q, hkv):
    """Blocks whose keys, then whose values, are many powers of two larger or smaller than those of the block before: the tokens that
    hold all the weight may be those with the smallest values."""
    import torch
    lens = [700, 330]
    rng, dev = make(gpu_api, 19, code, 128, "bf16", hkv, 1, lens, 704)
    powers = {"k": [0, 1, 4, 0, 6, 2, 7, 3, 0, 8, 5], "v": [0, 20, -100, 0, -100, -60, -100, 20, -30, -100, 0]}
    for kind, e in powers.items():
        by = np.exp2(np.array(e, dtype=np.float64))
        for b in range(2):
            for h in range(hkv):
                dev.ref[kind][b][h].s *= by[:len(dev.ref[kind][b][h].s)].astype(dev.ref[kind][b][h].s.dtype)
        dev.cache[kind].scales *= torch.from_numpy(by).float().cuda()
    run(gpu_api, rng, dev, 1, lens, n_q, spread=0.3)
    run(gpu_api, rng, dev, 1, lens, n_q, weights=True, causal=True, spread=0.3)


def test_a_nan_stays_in_its_row(gpu_api):
    import torch
    rng, dev = make(gpu_api, 21, E4M3, 128, "fp16", 2, 2, [300], 320)
    for n_q in (1, 50):
        q, _ = queries(rng, dev, 2, n_q)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        call = lambda x: gpu_api.nsn_q8_attention(dev.shape, x, dev.cache["k"], dev.cache["v"], i32([300]), 300, 0.1)  # noqa: E731
        clean, bad = call(q), q.clone()
        bad[0, n_q - 1, 1, 7] = float("nan")
        got = call(bad)
        torch.cuda.synchronize()
        assert torch.isnan(got[0, n_q - 1, 1]).all()
        got[0, n_q - 1, 1] = clean[0, n_q - 1, 1]
        assert torch.equal(got, clean)


@pytest.mark.parametrize("n_q,lens,heads", [(1, [2000, 700], 2), (6, [1500, 64], 2), (200, [900, 333], 2), (40, [900, 333], 64)])
def test_the_same_call_gives_the_same_bits_and_replays(gpu_api, n_q, lens, heads):
    """Twice eagerly, then captured into a graph and replayed between eager calls that share the workspace."""
    import torch
    api = gpu_api
    rng, dev = make(gpu_api, 31, INT8, 128, "bf16", heads, 4, lens, 2048)
    q, _ = queries(rng, dev, 4, n_q)
    ld = torch.tensor(lens, dtype=torch.int32).cuda()
    ws = torch.zeros(api.nsn_q8_workspace_bytes(dev.shape, api.NSN_OP_Q8_ATTENTION, 2, n_q, 2000), dtype=torch.uint8, device="cuda")
    w_in = torch.rand((2, heads, 2048), device="cuda")

    def call(out, lse, w):
        api.nsn_q8_attention(dev.shape, q, dev.cache["k"], dev.cache["v"], ld, 2000, 0.09, causal=True, weights_in=w_in, weights_out=w, out=out,
                             lse=lse, workspace=ws)
    make_out = lambda: (torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda"), torch.zeros_like(w_in))  # noqa: E731
    first, again, replay = make_out(), make_out(), make_out()
    call(*first)
    call(*again)
    torch.cuda.synchronize()
    for x, y in zip(first, again):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*replay)
    for _ in range(4):
        for x in replay:
            x.fill_(7)
        graph.replay()
        call(*again)
        torch.cuda.synchronize()
        for x, y, z in zip(first, again, replay):
            assert torch.equal(x, y)
            assert torch.equal(x, z) or (x.shape == w_in.shape and torch.equal(x[0, :, :lens[0]], z[0, :, :lens[0]]) and
                                         torch.equal(x[1, :, :lens[1]], z[1, :, :lens[1]]))


def test_one_workspace_serves_calls_of_different_sizes_in_turn(gpu_api):
    import torch
    api = gpu_api
    cases = []
    for seed, D, hkv, ratio, n_q, lens in ((1, 128, 2, 4, 1, [1500, 900]), (2, 64, 5, 1, 1, [777, 3]), (3, 128, 1, 8, 30, [640, 64]), (4, 128, 3, 2, 4, [1111, 1536]), (5, 64, 64, 3, 20, [300, 64])):
        rng, dev = make(api, seed, INT8, D, "fp16", hkv, ratio, lens, 1536)
        q, _ = queries(rng, dev, ratio, n_q)
        cases.append((dev, q, torch.tensor(lens, dtype=torch.int32).cuda(), max(lens)))
    need = max(api.nsn_q8_workspace_bytes(d.shape, api.NSN_OP_Q8_ATTENTION, 2, q.shape[1], n) for d, q, _, n in cases)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    call = lambda c, w: api.nsn_q8_attention(c[0].shape, c[1], c[0].cache["k"], c[0].cache["v"], c[2], c[3], 0.1, workspace=w)  # noqa: E731
    alone = [call(c, None) for c in cases]
    for _ in range(3):
        for c, x in zip(cases, alone):
            assert torch.equal(call(c, ws), x)


def test_on_a_stream_of_its_own(gpu_api):
    import torch
    rng, dev = make(gpu_api, 41, INT8, 128, "fp16", 2, 4, [600], 640)
    q, _ = queries(rng, dev, 4, 1)
    ld = torch.tensor([600], dtype=torch.int32).cuda()
    call = lambda: gpu_api.nsn_q8_attention(dev.shape, q, dev.cache["k"], dev.cache["v"], ld, 600, 0.1)  # noqa: E731
    ref = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = call()
    s.synchronize()
    assert torch.equal(ref, got)


def test_python_form_refuses_what_does_not_fit(gpu_api):
    import torch
    rng, dev = make(gpu_api, 43, INT8, 128, "fp16", 2, 2, [64], 128)
    q, _ = queries(rng, dev, 2, 1)
    ld = torch.tensor([64], dtype=torch.int32).cuda()
    call = lambda **kw: gpu_api.nsn_q8_attention(dev.shape, kw.pop("q", q), kw.pop("k", dev.cache["k"]), dev.cache["v"], kw.pop("lens", ld), 64, 0.1, **kw)  # noqa: E731
    call()
    for kw in (dict(q=q.bfloat16()), dict(q=q.cpu()), dict(q=q[:, :, :3]), dict(lens=ld.long()), dict(lens=ld[:0]), dict(out=q.float()),
               dict(lse=torch.zeros(2, device="cuda")), dict(weights_out=torch.zeros(3, device="cuda")),
               dict(k=gpu_api.Q8Cache(dev.cache["k"].codes[:, :1].contiguous(), dev.cache["k"].scales)),
               dict(q=torch.zeros((1, 1, 4, 256), dtype=torch.float16, device="cuda")[..., ::2])):
        with pytest.raises(AssertionError):
            call(**kw)
    wide = torch.zeros((1, 1, 4, 132), dtype=torch.float16, device="cuda")
    for kw in (dict(q=wide[..., 4:]), dict(q=wide[..., :128]), dict(workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(gpu_api.NsnError):
            call(**kw)


def test_a_serving_program_with_a_budget(gpu_api):
    """Prompt, chunk attention with weights, eviction, then decode steps that append, attend, add weights up and evict again: every
    attention output against the reference, which is carried along."""
    import torch
    from tests.test_gpu_q8_cache import evict_and_check
    api = gpu_api
    rng = np.random.default_rng(61)
    B, H, ratio, D, L, keep = 2, 2, 4, 128, 320, 128
    a, b = (Device(api, rng, INT8, D, H, B, L, 0, dtypes()["fp16"], ratio) for _ in range(2))
    lens = [300, 150]
    append(a, rng, [0, 0], lens, 300)
    w = torch.zeros((B, H, L), device="cuda")

    def attend(n_q, nq):
        q, ref_q = queries(rng, a, ratio, n_q)
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
        before = w.double().cpu().numpy()
        i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        api.nsn_q8_attention(a.shape, q, a.cache["k"], a.cache["v"], i32(lens), max(lens), 1 / np.sqrt(D), causal=True, q_lens=i32(nq),
                             weights_in=w, weights_out=w, out=out, lse=lse)
        torch.cuda.synchronize()
        compare(a, ref_q, out.double().cpu().numpy(), lse.cpu().numpy(), lens, nq, 1 / np.sqrt(D), True, ratio, np.zeros(q.shape),
                np.zeros(q.shape[:3], np.float32), w.cpu().numpy(), before, before.astype(np.float32))
    attend(300, lens)
    for step in range(3):
        at = w.cpu().numpy()
        evict_and_check(api, rng, a, b, lens, at, keep, 4, 32)
        new = np.zeros_like(at)
        for i in range(B):
            for h in range(H):
                sel = R.keep_of(at[i, h], lens[i], keep, 4, 32)
                new[i, h, :len(sel)] = at[i, h, sel]
        w = torch.from_numpy(new).cuda()
        lens = [min(n, keep) for n in lens]
        a, b = b, a
        for kind in "kv":
            b.noise[kind] = (b.cache[kind].codes.cpu().numpy().reshape(b.noise[kind][0].shape), b.cache[kind].scales.cpu().numpy())
        for _ in range(2):
            append(a, rng, lens, [1, 1], 1)
            lens = [n + 1 for n in lens]
            attend(1, [1, 1])


@pytest.mark.parametrize("code", [INT8, E4M3])
def test_missing_pages_of_many_heads(gpu_api, code):
    """The same where rows go 128 at a time."""
    lens = [512, 300, 130, 511, 64, 0, 400, 200]
    drop = [(0, 1, -1), (1, 0, 10 ** 9), (1, 2, 40), (2, 0, -7), (2, 1, -2 ** 31), (0, 3, 10), (6, 0, -1), (6, 1, -1), (6, 2, -1), (6, 3, -1)]
    rng, dev = make(gpu_api, 78, code, 128, "bf16", 16, 2, lens, 512, 128, drop=drop)
    for causal in (True, False):
        run(gpu_api, rng, dev, 2, lens, 30, causal=causal, weights=causal)


@pytest.mark.parametrize("batch,heads,n_q,ratio", [(8, 64, 33, 1), (40, 64, 1, 2), (16, 64, 3, 2), (70, 2, 1, 3), (131, 1, 2, 5), (70, 2, 35, 1), (130, 16, 20, 2)])
def test_many_sequences_and_heads(gpu_api, batch, heads, n_q, ratio):
    """More sequences than a wave has lanes, more units than runs, single tokens and chunks; lengths around the blocks, some of zero."""
    lens = [(37 * i + 5 * (i % 7)) % 140 if i % 11 else 0 for i in range(batch)]
    rng, dev = make(gpu_api, batch, INT8 if n_q % 2 else E4M3, 64, "fp16", heads, ratio, lens, 192)
    run(gpu_api, rng, dev, ratio, lens, n_q, causal=n_q > 1)
    nq = [(i * 7) % (n_q + 1) for i in range(batch)]
    run(gpu_api, rng, dev, ratio, lens, n_q, nq=nq, weights=heads < 4)
