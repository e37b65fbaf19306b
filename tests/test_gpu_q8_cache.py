"""Append to the 8-bit cache and eviction from it, against the format written out in numpy: codes and scales are equal, byte for byte."""
import numpy as np
import pytest

from tests import q8_reference as R

pytestmark = pytest.mark.gpu
INT8, E4M3 = R.INT8, R.E4M3


class Device:
    """A pair of caches whose places without a token hold random bytes, and the reference's units of them."""

    def __init__(self, api, rng, code, D, hkv, batch, max_len, page, dtype, ratio=1, drop=()):
        import torch
        self.api, self.code, self.D, self.hkv, self.batch, self.max_len, self.page = api, code, D, hkv, batch, max_len, page
        per = max_len // page if page else 0
        n_pages = batch * per + 3 if page else 0
        self.shape = api.make_q8_shape(D, hkv * ratio, hkv, max_len, page, n_pages, code, dtype)
        self.units = n_pages or batch
        self.tokens = page or max_len
        self.tables, self.cache, self.noise = {}, {}, {}
        order = rng.permutation(n_pages) if page else None
        for kind in "kv":
            raw = rng.integers(0, 256, (self.units, hkv, self.tokens * D), dtype=np.uint8)
            scales = np.full((self.units, hkv, self.tokens // 64), 7.5, np.float32)
            table = None
            if page:
                order = rng.permutation(n_pages)
                table = order[:batch * per].reshape(batch, per).astype(np.int32)
                for b, p, value in drop:
                    table[b, p] = value
            self.tables[kind], self.noise[kind] = table, (raw.copy(), scales.copy())
            self.cache[kind] = api.Q8Cache(torch.from_numpy(raw).cuda(), torch.from_numpy(scales).cuda(),
                                           None if table is None else torch.from_numpy(table).cuda())
        self.ref = {kind: [[R.Unit(code, D, max_len) for _ in range(hkv)] for _ in range(batch)] for kind in "kv"}

    def pages(self, kind, b, blk):
        """(unit, block inside it) of a sequence's 64-token block, or None."""
        if not self.page:
            return b, blk
        u = int(self.tables[kind][b, blk * 64 // self.page])
        return (u, blk % (self.page // 64)) if 0 <= u < self.units else None

    def expected(self, kind, written):
        """What the buffers hold when tokens [0, written[b]) of the reference have been written."""
        raw, scales = (x.copy() for x in self.noise[kind])
        off = R.offsets(kind, self.D, self.tokens)
        for b in range(self.batch):
            for h in range(self.hkv):
                unit = self.ref[kind][b][h]
                for blk in range(-(-written[b] // 64)):
                    at = self.pages(kind, b, blk)
                    if at is None:
                        continue
                    n = min(64, written[b] - 64 * blk)
                    rows = R.to_bytes(self.code, unit.c[64 * blk:64 * blk + n])
                    raw[at[0], h][off[64 * at[1]:64 * at[1] + n]] = rows
                    scales[at[0], h, at[1]] = unit.s[blk]
        return raw, scales

    def check(self, kind, written):
        raw, scales = self.expected(kind, written)
        got = self.cache[kind]
        assert np.array_equal(got.scales.cpu().numpy().view(np.uint32), scales.view(np.uint32)), kind
        assert np.array_equal(got.codes.cpu().numpy().reshape(raw.shape), raw), kind


def rows16(rng, dtype, *shape, spread=1.0):
    """16-bit values as a device tensor and in 64 bits."""
    import torch
    x = torch.from_numpy(rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape[:-1] + (1,)))).to(dtype)
    return x.cuda(), x.double().numpy()


def append(dev, rng, start, n, max_new, spread=1.0, transposed=False, change=None):
    import torch
    dt = dev.shape.dtype
    data = {}
    for kind in "kv":
        x, ref = rows16(rng, dt, dev.batch, dev.hkv, max_new, dev.D, spread=spread)
        if change is not None:
            change(x, kind)
            ref = x.double().cpu().numpy()
        if transposed:
            wide = torch.full((dev.batch, max_new, dev.hkv + 1, dev.D + 8), float("nan"), dtype=dt, device="cuda")
            wide[:, :, :dev.hkv, :dev.D] = x.transpose(1, 2)
            x = wide[:, :, :dev.hkv, :dev.D].transpose(1, 2)
        data[kind] = x
        for b in range(dev.batch):
            m = min(n[b], max_new)
            if start[b] >= 0 and m > 0:
                for h in range(dev.hkv):
                    dev.ref[kind][b][h].append(start[b], ref[b, h, :m])
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    dev.api.nsn_q8_append(dev.shape, data["k"], data["v"], i32(start), i32(n), dev.cache["k"], dev.cache["v"])
    torch.cuda.synchronize()


def dtypes():
    import torch
    return {"fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("io", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("code", [INT8, E4M3])
@pytest.mark.parametrize("page", [0, 64, 192])
def test_append_in_pieces(gpu_api, code, D, io, page):
    """Prompts of ragged lengths, then pieces from one token to several blocks that grow the scales of part-filled blocks."""
    rng = np.random.default_rng(100 * D + 10 * code + page)
    dev = Device(gpu_api, rng, code, D, 3, 4, 576, page, dtypes()[io])
    at = [0, 0, 0, 0]
    for i, n in enumerate(([1, 63, 64, 200], [1, 1, 1, 1], [62, 65, 0, 130], [1, 2, 3, 1], [200, 100, 1, 246])):
        append(dev, rng, at, n, max(n) + (i % 2), spread=0.5 * i, transposed=i % 2 == 1)
        at = [min(a + m, 576) for a, m in zip(at, n)]
        for kind in "kv":
            dev.check(kind, at)
    assert at[3] == 576   # (577 asked for: what lies beyond the cache is not written)


def test_append_goes_by_the_counts(gpu_api):
    """Counts above max_new, negative counts and starts, starts at the end and behind it: nothing but what is asked for is written."""
    rng = np.random.default_rng(5)
    dev = Device(gpu_api, rng, INT8, 128, 1, 6, 128, 0, dtypes()["fp16"])
    append(dev, rng, [0, -1, 0, 128, 2 ** 31 - 1, 100], [9, 3, -5, 4, 4, 0], 5)
    # sequence 0: five tokens (max_new); the others: none
    for kind in "kv":
        dev.check(kind, [5, 0, 0, 0, 0, 0])


@pytest.mark.parametrize("code", [INT8, E4M3])
def test_append_of_zeros_nan_and_infinities(gpu_api, code):
    import torch
    rng = np.random.default_rng(7)
    dev = Device(gpu_api, rng, code, 128, 2, 4, 128, 0, torch.bfloat16)

    def change(x, kind):
        x[0] = 0                                     # a block of zeros: scale 0
        x[1, :, 3, 5] = float("nan")
        x[1, :, 4, 6] = float("inf")
        x[1, :, 5, 7] = -float("inf")
        x[2] = float("inf")                          # no finite value at all
        x[3] = x[3] * 2.0 ** -120                    # around the least magnitude that has a scale
    append(dev, rng, [0] * 4, [70] * 4, 70, change=change)
    for kind in "kv":
        for b in (0, 2):
            for h in range(2):
                assert not dev.ref[kind][b][h].s.any() and not dev.ref[kind][b][h].c.any()
        dev.check(kind, [70] * 4)
    append(dev, rng, [70] * 4, [20] * 4, 20)         # then ordinary values into the same blocks
    for kind in "kv":
        dev.check(kind, [90] * 4)


@pytest.mark.parametrize("code", [INT8, E4M3])
def test_append_skips_pages_that_do_not_exist(gpu_api, code):
    rng = np.random.default_rng(8)
    dev = Device(gpu_api, rng, code, 64, 2, 2, 512, 128, dtypes()["fp16"], drop=[(0, 1, -1), (1, 2, 11), (1, 0, 2 ** 31 - 1)])
    append(dev, rng, [0, 5], [512, 400], 512)
    for kind in "kv":
        for h in range(2):   # tokens 0 .. 4 of sequence 1 were not there: its first page does not exist
            assert dev.pages(kind, 1, 0) is None
        dev.check(kind, [512, 405])


# ---- eviction ---------------------------------------------------------------------------------------------------------

def evict_and_check(api, rng, dev, to, lens, w, keep, first, recent, bound=None):
    """to: a Device that shares dev's buffers (paged) or has its own."""
    import torch
    B, H, D = dev.batch, dev.hkv, dev.D
    bound = max(lens) if bound is None else bound
    w_out = torch.full((B, H, dev.max_len), 3.25, device="cuda")
    kept, new_lens, moved = api.nsn_q8_evict(dev.shape, torch.from_numpy(w).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), bound,
                                             keep, dev.cache["k"], dev.cache["v"], to.cache["k"], to.cache["v"], first, recent,
                                             weights_out=w_out)
    torch.cuda.synchronize()
    kept, new_lens, moved = kept.cpu().numpy(), new_lens.cpu().numpy(), moved.cpu().numpy()
    n_new = [min(n, keep) for n in lens]
    assert new_lens.tolist() == n_new
    for b in range(B):
        for h in range(H):
            at = R.keep_of(w[b, h], lens[b], keep, first, recent)
            assert len(at) == n_new[b]
            assert np.array_equal(kept[b, h, :len(at)], at), (b, h)
            assert (kept[b, h, len(at):] == -1).all()
            ref = np.full(dev.max_len, 3.25, np.float32)
            ref[:bound] = 0
            ref[:len(at)] = w[b, h, at]
            assert np.array_equal(moved[b, h].view(np.uint32), ref.view(np.uint32))
            for kind in "kv":
                src, dst = dev.ref[kind][b][h], to.ref[kind][b][h]
                for blk in range(-(-len(at) // 64)):
                    sel = at[64 * blk:64 * blk + 64]
                    there = np.array([dev.pages(kind, b, t // 64) is not None for t in sel])
                    s = np.where(there, src.s[sel // 64], np.float32(0)).astype(np.float32)
                    lv = s.max()
                    ratio = s / lv if lv > 0 else np.zeros_like(s)
                    c = np.where(there[:, None], src.c[sel], 0.0).astype(np.float32)
                    dst.c[64 * blk:64 * blk + len(sel)] = R.round_code(dev.code, c * ratio.astype(np.float32)[:, None])
                    dst.s[blk] = lv
    for kind in "kv":
        to.check(kind, n_new)


def weights_of(rng, B, H, L, lens):
    w = np.exp(2 * rng.standard_normal((B, H, L))).astype(np.float32)
    w[rng.random((B, H, L)) < 0.3] = 0.0       # many equal ones
    for b in range(B):
        w[b, :, lens[b]:] = np.nan
    return w


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("code", [INT8, E4M3])
@pytest.mark.parametrize("lens,keep,first,recent", [([300, 0, 1, 65], 64, 4, 16), ([300, 299, 301, 64], 299, 0, 0), ([130, 200, 77, 70], 70, 70, 0),
                                                    ([130, 200, 77, 70], 70, 0, 70), ([320, 100, 200, 3], 1, 0, 0),
                                                    ([320, 319, 257, 129], 191, 3, 100), ([320, 63, 64, 65], 320, 10, 10)])
def test_evict(gpu_api, code, D, lens, keep, first, recent):
    rng = np.random.default_rng(1000 * D + keep)
    B, H, L = 4, 2, 320
    dev = Device(gpu_api, rng, code, D, H, B, L, 0, dtypes()["fp16"])
    append(dev, rng, [0] * B, lens, max(lens), spread=1.5)
    to = Device(gpu_api, rng, code, D, H, B, L, 0, dtypes()["fp16"])
    evict_and_check(gpu_api, rng, dev, to, lens, weights_of(rng, B, H, L, lens), keep, first, recent)


@pytest.mark.parametrize("code", [INT8, E4M3])
def test_evict_of_all_equal_of_infinite_and_of_nan_weights(gpu_api, code):
    rng = np.random.default_rng(11)
    lens, L = [3000, 2500, 2999, 1025, 1024], 3008
    dev = Device(gpu_api, rng, code, 64, 1, 5, L, 0, dtypes()["bf16"])
    append(dev, rng, [0] * 5, lens, max(lens))
    to = Device(gpu_api, rng, code, 64, 1, 5, L, 0, dtypes()["bf16"])
    w = weights_of(rng, 5, 1, L, lens)
    w[0] = 0.0
    w[1, 0, ::3], w[1, 0, 1::3], w[1, 0, 2::3] = np.inf, -np.inf, -0.0
    w[2, 0, ::2], w[2, 0, 1::4] = 0.0, -0.0
    w[3] = np.nan
    w[4, 0, ::2], w[4, 0, 1::2] = np.nan, -np.inf
    evict_and_check(gpu_api, rng, dev, to, lens, w, 1000, 0, 0, bound=L)


@pytest.mark.parametrize("code", [INT8, E4M3])
@pytest.mark.parametrize("page", [64, 128])
def test_evict_into_other_pages_of_the_same_pool(gpu_api, code, page):
    """Pages of the source and of the destination in one pool under two tables; a source page and a destination page that do not exist."""
    import torch
    rng = np.random.default_rng(12 + page)
    B, H, D, L = 2, 2, 128, 512
    dev = Device(gpu_api, rng, code, D, H, B, 2 * L, page, dtypes()["fp16"])
    half = L // page
    to = Device(gpu_api, rng, code, D, H, B, 2 * L, page, dtypes()["fp16"])
    for kind in "kv":      # the second half of each sequence's pages becomes the destination
        src = dev.tables[kind]
        dst = np.full_like(src, -1)
        dst[:, :half] = src[:, half:]
        src[:, half:] = -1
        src[0, 1], dst[1, half - 1] = -5, 10 ** 6
        codes, scales = dev.cache[kind].codes, dev.cache[kind].scales
        dev.cache[kind] = gpu_api.Q8Cache(codes, scales, torch.from_numpy(src.copy()).cuda())
        to.cache[kind] = gpu_api.Q8Cache(codes, scales, torch.from_numpy(dst.copy()).cuda())
        to.tables[kind] = dst
    lens = [500, 512]
    append(dev, rng, [0] * B, lens, 512)
    for kind in "kv":
        dev.check(kind, lens)
        to.noise[kind] = dev.expected(kind, lens)
    evict_and_check(gpu_api, rng, dev, to, lens, weights_of(rng, B, H, 2 * L, lens), 470, 4, 100)


def test_evict_then_append_then_evict(gpu_api):
    """The calls of a program that keeps its cache at a budget: the second eviction reads what the first one and an append left."""
    rng = np.random.default_rng(14)
    B, H, D, L = 2, 2, 128, 320
    a, b = (Device(gpu_api, rng, INT8, D, H, B, L, 0, dtypes()["fp16"]) for _ in range(2))
    lens = [320, 290]
    append(a, rng, [0, 0], lens, 320)
    for _ in range(3):
        evict_and_check(gpu_api, rng, a, b, lens, weights_of(rng, B, H, L, lens), 251, 4, 30)
        lens = [min(n, 251) for n in lens]
        append(b, rng, lens, [5, 17], 17)
        lens = [n + m for n, m in zip(lens, [5, 17])]
        for kind in "kv":
            b.check(kind, lens)
            a.noise[kind] = tuple(x.cpu().numpy().reshape(y.shape) for x, y in zip((a.cache[kind].codes, a.cache[kind].scales), a.noise[kind]))
        # the next destination keeps what it holds behind the tokens it is given
        a, b = b, a
        for kind in "kv":
            b.noise[kind] = (b.cache[kind].codes.cpu().numpy().reshape(b.noise[kind][0].shape), b.cache[kind].scales.cpu().numpy())


@pytest.mark.parametrize("length", [2048, 2049, 16384, 16385, 40001])
@pytest.mark.parametrize("kind", ["spread", "few values", "negative too"])
def test_evict_of_long_sequences(gpu_api, length, kind):
    """Around the lengths where the choice goes by another instance; weights over many powers of two, of few values, of both signs."""
    rng = np.random.default_rng(length)
    L = -(-length // 64) * 64
    lens = [length, length - 700]
    dev = Device(gpu_api, rng, E4M3, 64, 1, 2, L, 0, dtypes()["fp16"])
    append(dev, rng, [0, 0], lens, length)
    to = Device(gpu_api, rng, E4M3, 64, 1, 2, L, 0, dtypes()["fp16"])
    w = weights_of(rng, 2, 1, L, lens)
    if kind == "few values":
        w = np.round(w).clip(0, 3).astype(np.float32)
    elif kind == "negative too":
        w = (rng.standard_normal(w.shape) * 10.0 ** rng.integers(-30, 30, w.shape)).astype(np.float32)
    evict_and_check(gpu_api, rng, dev, to, lens, w, length // 3 + 1, 5, 99)


@pytest.mark.parametrize("code,D", [(INT8, 128), (E4M3, 64)])
def test_evict_of_many_sequences(gpu_api, code, D):
    """Enough blocks that a workgroup moves four; the last group is not full, nor is its last block."""
    rng = np.random.default_rng(88)
    lens = [4200, 4101, 4100, 4099, 64, 0, 4160, 4097]
    dev = Device(gpu_api, rng, code, D, 8, 8, 4224, 64, dtypes()["bf16"], drop=[(0, 3, -1)])
    append(dev, rng, [0] * 8, lens, max(lens))
    to = Device(gpu_api, rng, code, D, 8, 8, 4224, 64, dtypes()["bf16"], drop=[(1, 64, 10 ** 8), (2, 5, -2)])
    evict_and_check(gpu_api, rng, dev, to, lens, weights_of(rng, 8, 8, 4224, lens), 4100, 4, 500)
