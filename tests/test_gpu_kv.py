"""GPU: the paged key-value cache apart from a model (binding.KvCache) against plain evaluations in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ plain forms
def pow2(e):
    """2^e exactly (64-bit floats, integer e)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def quantised(x):
    """(codes as 64-bit values, E) of rows of x: E the smallest in -111..120 with max |finite x| <= 448 2^E; codes to nearest, ties to
    even, at steps of 2^-3 of their binade, of 2^-9 at least, and 240 2^120 at most; what is not finite: NaN."""
    x = x.detach().cpu().double()
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    e = torch.full(top.shape, -111, dtype=torch.long)
    for c in range(-111, 120):
        e = torch.where(top > 448.0 * 2.0 ** c, c + 1, e)
    y = torch.where(torch.isfinite(x), x, math.nan) / pow2(e).unsqueeze(-1)
    step = pow2(torch.frexp(torch.nan_to_num(y).abs().clamp(min=2.0 ** -6))[1] - 4)
    most = torch.where(e == 120, 240.0, 448.0).unsqueeze(-1)
    return torch.minimum(torch.maximum(torch.round(y / step) * step, -most), most), e


class Plain:
    """What a cache should hold, by (sequence, position): K, V [S][positions][H][D] in 64 bits."""

    def __init__(self, S, n, H, D, dtype):
        self.x = torch.zeros(2, S, n, H, D, dtype=torch.float64)
        self.dtype = dtype

    def append(self, k, v, pos, seq):
        for which, x in enumerate((k, v)):
            if self.dtype == "e4m3":
                c, e = quantised(x)
                y = c * pow2(e).unsqueeze(-1)
            else:
                y = x.detach().cpu().bfloat16().double()
            y = y.reshape(-1, *y.shape[-2:])
            for i, (s, p) in enumerate(zip(seq, pos)):
                if 0 <= s < self.x.shape[1] and 0 <= p < self.x.shape[2]:
                    self.x[which, s, p] = y[i]


def make(S, per_seq, H, D, page, dtype, seed, garbage=True):
    """A cache with its pages in random order and some to spare; what nobody wrote is random bytes."""
    from paper_2211_17192_amd import binding
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_pages = S * per_seq + 2
    table = torch.randperm(n_pages, generator=g, device="cuda")[:S * per_seq].view(S, per_seq).to(torch.int32)
    cache = binding.KvCache(table, n_pages, H, D, page_size=page, dtype=dtype)
    if garbage:
        cache.pool.view(torch.uint8).random_(0, 256, generator=g)
        if cache.exps is not None:
            cache.exps.random_(0, 256, generator=g)
    return cache, g


def normal(g, *shape, dtype="bf16", std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(TYPES[dtype])


def reference(plain, q, pos, scale, holes=None):
    """(out, lse, tolerance of out, tolerance of lse) in 64 bits."""
    S, R, H, D = q.shape
    K, V = plain.x.cuda()
    Hkv = K.shape[2]
    G = H // Hkv
    q = q.double()
    out, a = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((S, R, H), -math.inf, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(lse)
    for s in range(S):
        for r in range(R):
            n = min(int(pos[s, r]), K.shape[1] - 1) + 1
            if n <= 0:
                continue
            at = torch.arange(n, device="cuda")
            if holes is not None:
                at = at[~holes[s, :n].cuda()]
            if len(at) == 0:
                continue
            k, v = K[s, at].transpose(0, 1), V[s, at].transpose(0, 1)          # [Hkv, n, D]
            qq = q[s, r].view(Hkv, G, D)
            sc = torch.matmul(qq, k.transpose(1, 2)) * scale
            big = torch.matmul(qq.abs(), k.abs().transpose(1, 2)).amax(-1) * scale                 # bounds of the scores' terms
            p = torch.softmax(sc, -1)
            out[s, r] = torch.matmul(p, v).reshape(H, D)
            a[s, r] = torch.matmul(p, v.abs()).reshape(H, D)
            lse[s, r] = torch.logsumexp(sc, -1).reshape(H)
            # relative error of a weight: D + 8 roundings of 2^-24 in its score's terms (products are exact), the exponential's and the
            # exponent's 8; of a sum: one per addition, of which a lane's, the wavefronts' and the ranges' chains have n / 4 + 256 at most
            tol[s, r] = (2.0 ** -24 * ((D + 8) * big + 8 + n / 4 + 256)).reshape(H)
    return out, lse, a, tol


def check_attention(got, lse, q, plain, pos, scale=None, holes=None):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    ref, ref_lse, a, tol = reference(plain, q, pos, scale, holes)
    split = 2.0 ** -17 if q.dtype == torch.bfloat16 else 2.0 ** -24            # the weights as sums of bf16 numbers
    # a weight's error counts twice (in the sum and in its norm); the result is rounded once to its type
    bound = (2 * tol + split).unsqueeze(-1) * a * 1.0001 + ref.abs() * torch.finfo(q.dtype).eps / 2 * 1.0001 + 1e-30
    off = (got.double() - ref).abs()
    assert bool((off <= bound).all()), (float((off / bound).max()), float(off.max()))
    if lse is not None:
        none = ref_lse == -math.inf
        assert torch.equal(none, lse == -math.inf)
        off = torch.where(none, 0.0, (lse.double() - ref_lse).abs())
        assert bool((off <= 2 * tol + 2.0 ** -22 * (1 + torch.where(none, 0.0, ref_lse.abs()))).all()), float(off.max())


def fill(cache, g, lens, dtype="bf16", std=1.0):
    """Rows at positions 0 .. lens[s] - 1 of every sequence; returns the Plain of them."""
    n = max(max(lens), 1)
    plain = Plain(cache.n_seq, n, cache.n_kv_heads, cache.d_head, cache.dtype)
    k, v = (normal(g, cache.n_seq, n, cache.n_kv_heads, cache.d_head, dtype=dtype, std=std) for _ in range(2))
    k[..., 3] *= 8                                     # an outlying channel
    pos = torch.tensor([[p if p < L else -1 for p in range(n)] for L in lens], dtype=torch.int32, device="cuda")
    cache.append(k, v, pos)
    plain.append(k, v, pos.flatten().tolist(), [s for s in range(cache.n_seq) for _ in range(n)])
    return plain


# ------------------------------------------------------------------ rows in and out
SHAPES = [(1, 32, 16), (2, 64, 16), (8, 128, 16), (3, 128, 64), (12, 64, 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("H,D,page", SHAPES)
def test_rows_in_and_out(dtype, cache_dtype, H, D, page):
    """What is read back is what the definition says, to the bit; nothing else in the pool has changed; absent rows read as zeros."""
    S, per_seq, n = 3, 4, 37
    cache, g = make(S, per_seq, H, D, page, cache_dtype, 1)
    before, exps_before = cache.pool.clone(), None if cache.exps is None else cache.exps.clone()
    x = normal(g, n, 2, H, D, dtype=dtype) * torch.exp(3 * torch.randn(n, 2, H, 1, generator=g, device="cuda")).to(TYPES[dtype])
    x[0], x[1, 0, 0, 5], x[2] = 0.0, 1e30, x[2] * 1e-33
    k, v = x[:, 0], x[:, 1]                            # views with strides
    place = torch.randperm(S * per_seq * page, generator=g, device="cuda")[:n]
    seq, pos = (place // (per_seq * page)).to(torch.int32), (place % (per_seq * page)).to(torch.int32)
    pos[3], pos[4], pos[5], pos[6], seq[7], seq[8] = -1, per_seq * page, -2 ** 31, 2 ** 31 - 1, S, -1
    cache.append(k, v, pos, seq=seq)
    plain = Plain(S, per_seq * page, H, D, cache_dtype)
    plain.append(k, v, pos.tolist(), seq.tolist())
    gone = torch.zeros(n, dtype=torch.bool)
    gone[3:9] = True
    s, p = seq.cpu().long().clamp(0, S - 1), pos.cpu().long().clamp(0, per_seq * page - 1)
    for out in ("bf16", "f32"):
        got = cache.read(pos, seq=seq, dtype=TYPES[out])
        for which in range(2):
            want = torch.where(gone[:, None, None], 0.0, plain.x[which, s, p])
            assert torch.equal(got[which].cpu().double(), want), (out, which)
    keep = torch.ones(cache.pool.shape[0], page, dtype=torch.bool, device="cuda")
    keep[cache.page_table[s.cuda(), p.cuda() // page].long()[~gone], (p.cuda() % page)[~gone]] = False
    same = (cache.pool.view(torch.uint8) == before.view(torch.uint8)).view(*cache.pool.shape[:4], -1).all(-1)
    assert bool(same.permute(0, 3, 1, 2)[keep].all())
    if exps_before is not None:
        assert bool((cache.exps == exps_before).permute(0, 3, 1, 2)[keep].all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("S,R,H,D", [(3, 1500, 8, 128), (5, 3001, 12, 64), (2, 9000, 9, 32), (16, 2001, 8, 128)])
def test_many_rows_are_what_few_at_a_time_are(dtype, cache_dtype, S, R, H, D):
    """Padded batches of 8 MB and more against pieces of 100 rows, which the tests above pin: the whole pool, and what is read of it."""
    from paper_2211_17192_amd import binding
    cache, g = make(S, -(-R // 64), H, D, 64, cache_dtype, 25)
    other = binding.KvCache(cache.page_table, cache.pool.shape[0], H, D, page_size=64, dtype=cache_dtype, pool=cache.pool.clone(), exps=None if cache.exps is None else cache.exps.clone())
    x = normal(g, S, R, 2, H, D, dtype=dtype)
    k, v = x[:, :, 0], x[:, :, 1]
    pos = torch.arange(R, dtype=torch.int32, device="cuda").repeat(S, 1).contiguous()
    for s in range(S):
        pos[s, R - R * s // S:] = -1                   # shorter sequences
    pos[0, ::7] = -1
    cache.append(k, v, pos)
    for r in range(0, R, 100):
        other.append(k[:, r:r + 100].contiguous(), v[:, r:r + 100].contiguous(), pos[:, r:r + 100].contiguous())
    assert torch.equal(cache.pool.view(torch.uint8), other.pool.view(torch.uint8))
    if cache.exps is not None:
        assert torch.equal(cache.exps, other.exps)
    got = cache.read(pos, dtype=TYPES[dtype])
    for r in range(0, R, 700):
        few = other.read(pos[:, r:r + 100].contiguous(), dtype=TYPES[dtype])
        for a, b in zip(got, few):
            assert torch.equal(a[:, r:r + 100], b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_magnitude_and_tie(dtype):
    """Rows of every binade, with ties, the largest finite numbers, subnormals, zeros of both signs."""
    cache, g = make(1, 40, 1, 32, 16, "e4m3", 2)
    t = TYPES[dtype]
    e = torch.arange(-149, 128, device="cuda")
    scale = torch.cat([pow2(e.clamp(min=-149)).to(torch.float32), torch.tensor([torch.finfo(t).max], device="cuda")])
    m = torch.tensor([1.0, 1.75, 1.7578125, 1.9921875, 0.0, -0.0, 0.5625, 0.53125, 0.59375, -0.65625, 2.0 ** -8, 2.0 ** -9, 2.0 ** -14, 2.0 ** -15, 2.0 ** -16,
                      2.0 ** -17, 2.0 ** -18, 2.0 ** -19, 3 * 2.0 ** -19, 0.99, -1.0, 0.3, 0.7, -0.1, 1 / 3, 0.8125, 0.84375, 0.90625, 0.9375, 0.96875, 0.015625, 0.1], device="cuda")
    rows = [(scale[:, None] * (m[None, :] * f)).to(t) for f in (1.0, 0.5, 0.499)]
    x = torch.cat(rows)[:640].view(-1, 1, 32)
    x = torch.where(torch.isfinite(x), x, torch.tensor(1.0, device="cuda", dtype=t))
    pos = torch.arange(len(x), dtype=torch.int32, device="cuda")[None]
    cache.append(x[None], -x[None], pos)
    k, v = cache.read(pos, dtype=torch.float32)
    c, ex = quantised(x)
    want = c * pow2(ex).unsqueeze(-1)
    assert torch.equal(k.cpu()[0].double(), want) and torch.equal(v.cpu()[0].double(), -want)


@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
def test_what_is_not_finite_is_kept_as_such(cache_dtype):
    cache, g = make(1, 2, 2, 64, 16, cache_dtype, 3)
    x = normal(g, 1, 4, 2, 64)
    x[0, 1, 0, 7], x[0, 1, 0, 8], x[0, 2, 1, 0], x[0, 3] = math.nan, math.inf, -math.inf, math.nan
    pos = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    cache.append(x, x, pos)
    k, _ = cache.read(pos)
    if cache_dtype == "bf16":
        assert torch.equal(k.view(torch.int16), x.view(torch.int16))
        return
    bad = ~torch.isfinite(x)
    assert torch.equal(torch.isnan(k), bad)
    c, e = quantised(x)
    want = (c * pow2(e).unsqueeze(-1)).cuda()
    assert torch.equal(k.double()[~bad], want[~bad])


def test_pages_outside_the_pool_are_neither_written_nor_read():
    cache, g = make(2, 3, 2, 32, 16, "e4m3", 4)
    cache.page_table[0, 1], cache.page_table[1, 2] = -1, cache.pool.shape[0]
    before = cache.pool.clone()
    x = normal(g, 2, 48, 2, 32)
    pos = torch.arange(48, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()
    cache.append(x, x, pos)
    k, v = cache.read(pos)
    c, e = quantised(x)
    want = (c * pow2(e).unsqueeze(-1)).cuda()
    want[0, 16:32], want[1, 32:48] = 0.0, 0.0
    assert torch.equal(k.double(), want) and torch.equal(v.double(), want)
    used = set(cache.page_table[0].tolist()) | set(cache.page_table[1].tolist())
    for p in range(before.shape[0]):
        if p not in used:
            assert torch.equal(cache.pool[p], before[p])


def test_no_rows_and_rows_without_a_position_list():
    from paper_2211_17192_amd import binding
    cache, g = make(2, 2, 2, 64, 16, "e4m3", 5)
    before = cache.pool.clone()
    empty = torch.empty(2, 0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(empty, empty, torch.empty(2, 0, dtype=torch.int32, device="cuda"))
    assert cache.read(torch.empty(2, 0, dtype=torch.int32, device="cuda"))[0].shape == (2, 0, 2, 64)
    assert torch.equal(cache.pool, before)
    # the C entry without positions: 0, 1, .. of each sequence
    x = normal(g, 2, 5, 2, 64)
    rows = binding._KvRows(x.data_ptr(), x.data_ptr(), 128, 64, 128, 64, binding.SD_BF16)
    assert binding.lib.sd_kv_append(cache._ref, rows, None, None, 10, binding._stream()) == binding.SD_OK
    k, _ = cache.read(torch.arange(5, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous())
    c, e = quantised(x)
    assert torch.equal(k.cpu().double(), c * pow2(e).unsqueeze(-1))


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("H,Hkv,D,page", [(2, 2, 32, 16), (4, 1, 64, 16), (8, 2, 128, 16), (3, 3, 128, 64), (6, 2, 64, 128), (8, 4, 32, 32)])
def test_attention_over_ragged_contexts(dtype, cache_dtype, H, Hkv, D, page):
    """Lengths around tiles, steps, turns and ranges; sequences with fewer rows than others, and with none."""
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 300, 511, 700, 3, 40]
    S, R = len(lens), 3
    cache, g = make(S, -(-800 // page), Hkv, D, page, cache_dtype, 6)
    plain = fill(cache, g, lens, dtype=dtype)
    q = normal(g, S, R, H, D, dtype=dtype, std=2.0)
    pos = torch.tensor([[L - R + r for r in range(R)] for L in lens], dtype=torch.int32, device="cuda")       # (negative where L < R)
    pos[9, 1], pos[12, 0], pos[15] = -1, 0, -1
    for max_len in (None, 700):
        lse = torch.empty(S, R, H, device="cuda")
        out = cache.attention(q, pos, max_len=max_len, lse=lse)
        check_attention(out, lse, q, plain, pos)
    empty = pos < 0
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())


@pytest.mark.parametrize("H,Hkv,R", [(32, 8, 1), (32, 8, 5), (32, 8, 8), (4, 1, 16), (16, 16, 16), (40, 1, 2), (9, 3, 11), (64, 64, 1)])
@pytest.mark.parametrize("dtype,cache_dtype", [("bf16", "e4m3"), ("f32", "bf16"), ("f32", "e4m3"), ("bf16", "bf16")])
def test_attention_over_every_number_of_rows(dtype, cache_dtype, H, Hkv, R):
    """One and two row tiles, several groups of them, contexts of several ranges."""
    D = 64 if H == 64 else 128
    lens = [1500, 5000]
    cache, g = make(2, 5120 // 16, Hkv, D, 16, cache_dtype, 7)
    plain = fill(cache, g, lens, dtype=dtype)
    q = normal(g, 2, R, H, D, dtype=dtype, std=2.0)
    pos = torch.tensor([[L - R + r for r in range(R)] for L in lens], dtype=torch.int32, device="cuda")
    lse = torch.empty(2, R, H, device="cuda")
    out = cache.attention(q, pos, max_len=5000, lse=lse)
    check_attention(out, lse, q, plain, pos)
    assert torch.equal(out, cache.attention(q, pos, max_len=5000))


@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,H,Hkv,R", [(2, 32, 8, 1), (2, 32, 8, 5), (2, 32, 8, 9), (8, 8, 8, 16), (8, 16, 8, 17)])
def test_attention_cut_for_long_contexts(dtype, cache_dtype, S, H, Hkv, R):
    """Calls that are cut for contexts of 40000, whatever theirs are: one and two tiles, one and several groups; table entries behind a context are anything."""
    D, max_len = 128, 40000
    lens = [700, 33, 5, 1000, 1, 64, 257, 500][:S]
    cache, g = make(S, 64, Hkv, D, 16, cache_dtype, 20)
    wide = torch.randint(-5, cache.pool.shape[0] + 5, (S, 2500), dtype=torch.int32, device="cuda", generator=g)
    wide[:, :64] = cache.page_table
    plain = fill(cache, g, lens, dtype=dtype)
    cache = type(cache)(wide, cache.pool.shape[0], Hkv, D, dtype=cache_dtype, pool=cache.pool, exps=cache.exps)
    q = normal(g, S, R, H, D, dtype=dtype, std=2.0)
    pos = torch.tensor([[L - R + r for r in range(R)] for L in lens], dtype=torch.int32, device="cuda")
    pos[1, 0] = 32
    lse = torch.empty(S, R, H, device="cuda")
    out = cache.attention(q, pos, max_len=max_len, lse=lse)
    check_attention(out, lse, q, plain, pos)
    assert torch.equal(out, cache.attention(q, pos, max_len=max_len))


@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,page", [(32, 16), (64, 16), (64, 64)])
@pytest.mark.parametrize("R", [1, 5])
def test_small_heads_cut_for_long_contexts(dtype, cache_dtype, D, page, R):
    """Rows of 32, 64 and 128 bytes in calls whose contexts may be 60000 long: one tile and two."""
    S, H, Hkv, max_len = 5, 32, 8, 60000
    lens = [700, 33, 5, 1000, 257]
    cache, g = make(S, 1024 // page, Hkv, D, page, cache_dtype, 22)
    plain = fill(cache, g, lens, dtype=dtype)
    wide = torch.zeros(S, -(-max_len // page), dtype=torch.int32, device="cuda")
    wide[:, :1024 // page] = cache.page_table
    cache = type(cache)(wide, cache.pool.shape[0], Hkv, D, page_size=page, dtype=cache_dtype, pool=cache.pool, exps=cache.exps)
    q = normal(g, S, R, H, D, dtype=dtype, std=2.0)
    pos = torch.tensor([[L - R + r for r in range(R)] for L in lens], dtype=torch.int32, device="cuda")
    lse = torch.empty(S, R, H, device="cuda")
    check_attention(cache.attention(q, pos, max_len=max_len, lse=lse), lse, q, plain, pos)


@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv,D,R,max_len", [(32, 8, 128, 1, 700), (32, 8, 128, 5, 2600), (64, 32, 64, 1, 1200), (16, 16, 32, 3, 3000)])
def test_attention_with_eight_wavefronts(dtype, cache_dtype, H, Hkv, D, R, max_len):
    lens = [700, 512, 257, 256, 255, 1, 33, 600]
    cache, g = make(8, -(-max_len // 16), Hkv, D, 16, cache_dtype, 21)
    plain = fill(cache, g, lens, dtype=dtype)
    q = normal(g, 8, R, H, D, dtype=dtype, std=2.0)
    pos = torch.tensor([[L - R + r for r in range(R)] for L in lens], dtype=torch.int32, device="cuda")
    lse = torch.empty(8, R, H, device="cuda")
    check_attention(cache.attention(q, pos, max_len=max_len, lse=lse), lse, q, plain, pos)


@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("n", [66000, 131072])
def test_attention_over_a_very_long_context(cache_dtype, n):
    cache, g = make(1, n // 64 + 1, 2, 64, 64, cache_dtype, 8)
    plain = Plain(1, n, 2, 64, "bf16")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    k, v = (normal(g, 1, n, 2, 64) for _ in range(2))
    cache.append(k, v, pos)
    plain.x = torch.stack(cache.read(pos, dtype=torch.float32)).cpu().double()           # (pinned by the tests above)
    q = normal(g, 1, 4, 4, 64, std=3.0)
    at = torch.tensor([[n - 4, n - 3, n - 2, n - 1]], dtype=torch.int32, device="cuda")
    lse = torch.empty(1, 4, 4, device="cuda")
    check_attention(cache.attention(q, at, max_len=n, lse=lse), lse, q, plain, at)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("S,H,Hkv,D,R,top", [(33, 32, 8, 128, 5, 90), (20, 16, 4, 128, 13, 200), (2, 4, 2, 32, 1, 9000), (3, 12, 12, 64, 6, 2100), (40, 4, 2, 32, 2, 1300)])
def test_attention_with_many_groups_and_many_ranges(dtype, cache_dtype, S, H, Hkv, D, R, top):
    """More groups of rows than CUs; short rows in many ranges, or with eight wavefronts."""
    g = torch.Generator().manual_seed(24)
    lens = [int(n) for n in torch.randint(1, top + 1, (S,), generator=g)]
    lens[0] = top
    cache, g = make(S, -(-top // 16), Hkv, D, 16, cache_dtype, 24)
    plain = fill(cache, g, lens, dtype=dtype)
    q = normal(g, S, R, H, D, dtype=dtype, std=2.0)
    pos = torch.tensor([[L - R + r for r in range(R)] for L in lens], dtype=torch.int32, device="cuda")
    lse = torch.empty(S, R, H, device="cuda")
    out = cache.attention(q, pos, max_len=top, lse=lse)
    check_attention(out, lse, q, plain, pos)
    assert torch.equal(out, cache.attention(q, pos, max_len=top))


def test_many_rows_cut_for_the_longest_contexts():
    """520 groups of rows times 128 ranges of keys."""
    from paper_2211_17192_amd import binding
    n, R = 300, 4160
    cache, g = make(1, 32, 1, 128, 16, "e4m3", 23)
    plain = fill(cache, g, [n])
    wide = torch.zeros(1, binding.SD_KV_MAX_LEN // 16, dtype=torch.int32, device="cuda")
    wide[:, :32] = cache.page_table
    cache = type(cache)(wide, cache.pool.shape[0], 1, 128, pool=cache.pool, exps=cache.exps)
    q = normal(g, 1, R, 4, 128, std=2.0)
    pos = torch.randint(-1, n, (1, R), dtype=torch.int32, device="cuda", generator=g)
    lse = torch.empty(1, R, 4, device="cuda")
    out = cache.attention(q, pos, max_len=binding.SD_KV_MAX_LEN, lse=lse)
    check_attention(out, lse, q, plain, pos)


@pytest.mark.parametrize("scale", [0.01, 1.0, 20.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_with_flat_and_peaked_weights(scale, dtype):
    cache, g = make(2, 20, 2, 64, 32, "e4m3", 9)
    plain = fill(cache, g, [600, 33], dtype=dtype)
    q = normal(g, 2, 2, 4, 64, dtype=dtype)
    pos = torch.tensor([[598, 599], [31, 32]], dtype=torch.int32, device="cuda")
    lse = torch.empty(2, 2, 4, device="cuda")
    check_attention(cache.attention(q, pos, scale=scale, lse=lse), lse, q, plain, pos, scale=scale)


@pytest.mark.parametrize("cache_dtype", ["e4m3", "bf16"])
@pytest.mark.parametrize("R,max_len", [(4, None), (20, None), (12, 140000), (20, 140000)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_rows_are_not_reached_by_what_they_do_not_see(cache_dtype, R, max_len, bad):
    """K and V of the last rows are not finite: rows before them are as if they were, rows that see them are not finite either."""
    n = 600
    cache, g = make(2, 48, 2, 128, 16, cache_dtype, 10)
    plain = fill(cache, g, [n, n])
    if max_len is not None:                            # (two tiles of rows)
        table = torch.zeros(2, max_len // 16, dtype=torch.int32, device="cuda")
        table[:, :48] = cache.page_table
        cache = type(cache)(table, cache.pool.shape[0], 2, 128, dtype=cache_dtype, pool=cache.pool, exps=cache.exps)
    q = normal(g, 2, R, 4, 128)
    pos = torch.tensor([[n - R + r for r in range(R)]] * 2, dtype=torch.int32, device="cuda")
    pos[1, 1] = -1
    good = cache.attention(q, pos)
    x = normal(g, 2, 1, 2, 128)
    x[:, :, :, 5], x[:, :, :, 100] = bad, bad
    for part in ("k", "v"):
        last = torch.tensor([[n - 2], [n - 2]], dtype=torch.int32, device="cuda")
        k, v = (x if part == p else normal(torch.Generator(device="cuda").manual_seed(1), 2, 1, 2, 128) for p in "kv")
        cache.append(k, v, last)
        lse = torch.empty(2, R, 4, device="cuda")
        out = cache.attention(q, pos, lse=lse)
        assert torch.equal(out[:, :R - 2], good[:, :R - 2])
        if part == "k":
            assert not bool(torch.isfinite(out[:, R - 2:]).any()) or math.isinf(bad)     # (an infinite score may be minus infinity: no weight)
            if math.isnan(bad):
                assert bool(torch.isnan(out[:, R - 2:]).all())
        else:
            seen = torch.isfinite(out[:, R - 2:])
            assert not bool(seen[..., [5, 100]].any()) and bool(seen[..., [0, 4, 6, 99, 101, 127]].all())
    assert bool((out[1, 1] == 0).all()) and bool((lse[1, 1] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_without_a_page_are_not_seen(dtype):
    lens = [200, 64, 30, 700]
    cache, g = make(4, 48, 2, 64, 16, "e4m3", 11)
    plain = fill(cache, g, lens)
    holes = torch.zeros(4, 768, dtype=torch.bool)
    for s, page, entry in ((0, 0, -1), (0, 7, 10 ** 9), (1, 3, cache.pool.shape[0]), (2, 0, -5), (2, 1, -5), (3, 20, -1), (3, 43, -1)):
        cache.page_table[s, page] = entry
        holes[s, 16 * page:16 * page + 16] = True
    q = normal(g, 4, 2, 4, 64, dtype=dtype)
    pos = torch.tensor([[L - 2, L - 1] for L in lens], dtype=torch.int32, device="cuda")
    lse = torch.empty(4, 2, 4, device="cuda")
    out = cache.attention(q, pos, lse=lse)
    check_attention(out, lse, q, plain, pos, holes=holes)
    assert bool((out[2] == 0).all())


def test_positions_beyond_max_len_and_the_table():
    cache, g = make(2, 20, 2, 64, 16, "e4m3", 12)
    plain = fill(cache, g, [320, 320])
    q = normal(g, 2, 2, 4, 64)
    pos = torch.tensor([[99, 2 ** 31 - 1], [320, 100]], dtype=torch.int32, device="cuda")
    for max_len, top in ((None, 319), (4096, 319), (100, 99), (1, 0)):
        out = cache.attention(q, pos, max_len=max_len)
        check_attention(out, None, q, plain, pos.clamp(max=top))


def test_queries_with_strides_and_fused_rows():
    """k, v and q as parts of one projection's output; q with heads in front of rows."""
    S, R, H, Hkv, D = 3, 4, 8, 2, 64
    cache, g = make(S, 4, Hkv, D, 16, "e4m3", 13)
    plain = Plain(S, 64, Hkv, D, "e4m3")
    x = normal(g, S, R, H + 2 * Hkv, D)
    q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
    pos = torch.arange(R, dtype=torch.int32, device="cuda").repeat(S, 1).contiguous()
    cache.append(k, v, pos)
    plain.append(k, v, pos.flatten().tolist(), [s for s in range(S) for _ in range(R)])
    out = cache.attention(q, pos)
    check_attention(out, None, q, plain, pos)
    turned = q[:1].transpose(1, 2).contiguous().transpose(1, 2)
    one = type(cache)(cache.page_table[:1].contiguous(), cache.pool.shape[0], Hkv, D, pool=cache.pool, exps=cache.exps)
    assert torch.equal(one.attention(turned, pos[:1].contiguous(), max_len=64), one.attention(q[:1].contiguous(), pos[:1].contiguous(), max_len=64))


def test_far_pages():
    """A pool of more than 2^32 bytes: rows at its end."""
    from paper_2211_17192_amd import binding
    n_pages = 70000                                    # 64 positions x 8 heads x 128 x 2: 131072 bytes a page, 9.2 GB
    pool = torch.empty(n_pages, 2, 8, 64, 128, dtype=torch.uint8, device="cuda")
    exps = torch.empty(n_pages, 2, 8, 64, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_pages - 1, 3, n_pages - 7]], dtype=torch.int32, device="cuda")
    cache = binding.KvCache(table, n_pages, 8, 128, page_size=64, pool=pool, exps=exps)
    g = torch.Generator(device="cuda").manual_seed(14)
    plain = fill(cache, g, [190])
    q = normal(g, 1, 2, 16, 128)
    pos = torch.tensor([[188, 189]], dtype=torch.int32, device="cuda")
    check_attention(cache.attention(q, pos), None, q, plain, pos)
    at = torch.arange(190, dtype=torch.int32, device="cuda")[None]
    assert torch.equal(cache.read(at)[1].cpu()[0].double(), plain.x[1, 0])


def test_other_sequences_do_not_matter_and_results_repeat():
    lens = [900, 300, 2000]
    cache, g = make(3, 126, 2, 128, 16, "e4m3", 15)
    fill(cache, g, lens)
    q = normal(g, 3, 2, 8, 128)
    pos = torch.tensor([[L - 2, L - 1] for L in lens], dtype=torch.int32, device="cuda")
    scratch = cache.attention_scratch(8, 2)
    first = cache.attention(q, pos, scratch=scratch)
    for _ in range(20):
        assert torch.equal(cache.attention(q, pos, scratch=scratch), first)
    q2, pos2 = q.clone(), pos.clone()
    q2[1], pos2[1] = 0, -1
    again = cache.attention(q2, pos2, scratch=scratch)
    assert torch.equal(again[[0, 2]], first[[0, 2]])
    assert int(scratch[:4 * 65536].sum()) == 0         # (the tickets)


def test_on_another_stream_and_with_scratch_of_other_calls():
    cache, g = make(4, 126, 2, 64, 16, "e4m3", 16)
    plain = fill(cache, g, [2000, 1, 77, 1200])
    scratch = cache.attention_scratch(16, 9, max_len=2016)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for R, H, max_len in ((9, 16, 2016), (1, 2, 2000), (3, 8, 2016), (2, 2, 64), (1, 16, 1200)):
            q = normal(g, 4, R, H, 64)
            pos = torch.tensor([[L - R + r for r in range(R)] for L in (2000, 1, 77, 1200)], dtype=torch.int32, device="cuda")
            check_attention(cache.attention(q, pos, max_len=max_len, scratch=scratch), None, q, plain, pos.clamp(max=max_len - 1))
    torch.cuda.current_stream().wait_stream(side)


def test_captured_and_replayed():
    """A step (append, attention) as a graph: replayed with other rows, positions and page tables, eager calls in between on the same scratch; a
    second graph shares the scratch."""
    S, R, H, Hkv, D, n = 3, 2, 8, 2, 128, 1500
    cache, g = make(S, 100, Hkv, D, 16, "e4m3", 17)
    plain = fill(cache, g, [n, 700, 40])
    lens = [n, 700, 40]
    grown = Plain(S, 1600, Hkv, D, "e4m3")
    grown.x[:, :, :n] = plain.x
    q, k, v = normal(g, S, R, H, D), normal(g, S, R, Hkv, D), normal(g, S, R, Hkv, D)
    pos = torch.zeros(S, R, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(S, R, H, device="cuda")
    scratch = cache.attention_scratch(H, R, max_len=1600)

    def step():
        cache.append(k, v, pos)
        cache.attention(q, pos, max_len=1600, out=out, lse=lse, scratch=scratch)

    def attend_again():
        cache.attention(q, pos, max_len=1600, out=out, lse=lse, scratch=scratch)

    graphs = []
    for what in (step, attend_again):
        pos.copy_(torch.tensor([[L + r for r in range(R)] for L in lens], dtype=torch.int32))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            what()
        graphs.append(graph)
    for it in range(4):
        for x, y in ((q, normal(g, S, R, H, D)), (k, normal(g, S, R, Hkv, D)), (v, normal(g, S, R, Hkv, D))):
            x.copy_(y)
        at = [[L + r for r in range(R)] for L in lens]
        if it == 2:
            at[1][1] = -1
        pos.copy_(torch.tensor(at, dtype=torch.int32))
        graphs[0].replay()
        grown.append(k, v, [p for ps in at for p in ps], [s for s in range(S) for _ in range(R)])
        check_attention(out, lse, q, grown, pos)
        first = out.clone()
        out.zero_()
        graphs[1].replay()
        assert torch.equal(out, first)
        attend_again()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        lens = [L + 1 + min((it + s) % R, sum(p >= 0 for p in at[s]) - 1) for s, L in enumerate(lens)]   # rows that were not accepted are overwritten


def test_a_decoding_loop():
    """Prompts in, then verify steps of gamma + 1 rows with roll-backs, for sequences of their own lengths; the whole cache read back at the end."""
    S, H, Hkv, D, gamma = 4, 8, 2, 64, 3
    cache, g = make(S, 20, Hkv, D, 16, "e4m3", 18)
    lens = [100, 1, 17, 260]
    plain = Plain(S, 320, Hkv, D, "e4m3")
    first = fill(cache, g, lens, dtype="f32")
    plain.x[:, :, :260] = first.x
    scratch = cache.attention_scratch(H, gamma + 1)
    for it in range(5):
        pos = torch.tensor([[L + r for r in range(gamma + 1)] for L in lens], dtype=torch.int32, device="cuda")
        x = normal(g, S, gamma + 1, H + 2 * Hkv, D, dtype="f32")
        q, k, v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
        cache.append(k, v, pos)
        plain.append(k, v, pos.flatten().tolist(), [s for s in range(S) for _ in range(gamma + 1)])
        check_attention(cache.attention(q, pos, scratch=scratch), None, q, plain, pos)
        lens = [L + 1 + (it * 7 + s) % (gamma + 1) for s, L in enumerate(lens)]
    at = torch.tensor([[p if p < L else -1 for p in range(320)] for L in lens], dtype=torch.int32, device="cuda")
    got = cache.read(at, dtype=torch.float32)
    for s, L in enumerate(lens):
        for which in range(2):
            assert torch.equal(got[which][s, :L].cpu().double(), plain.x[which, s, :L])
            assert bool((got[which][s, L:] == 0).all())


# ------------------------------------------------------------------ refusals on a GPU (the C entry's own: test_kv.py)
def test_refusals_of_the_binding():
    from paper_2211_17192_amd import binding
    cache, g = make(2, 4, 2, 64, 16, "e4m3", 19)
    k, pos = normal(g, 2, 3, 2, 64), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    q = normal(g, 2, 3, 4, 64)
    bad = [
        lambda: binding.KvCache(cache.page_table, 3, 2, 64, dtype="fp8"),
        lambda: binding.KvCache(cache.page_table.long(), 3, 2, 64),
        lambda: binding.KvCache(cache.page_table.cpu(), 3, 2, 64),
        lambda: binding.KvCache(cache.page_table, 3, 2, 64, pool=cache.pool),
        lambda: binding.KvCache(cache.page_table, 0, 2, 64),
        lambda: binding.KvCache(cache.page_table, 3, 2, 48).append(normal(g, 2, 3, 2, 48), normal(g, 2, 3, 2, 48), pos),
        lambda: cache.append(k.half(), k.half(), pos),
        lambda: cache.append(k, k.float(), pos),
        lambda: cache.append(k[:, :2], k[:, :2], pos),
        lambda: cache.append(k, k, pos.long()),
        lambda: cache.append(k, k, pos.flatten()),
        lambda: cache.append(k, k, pos, seq=pos[:1].contiguous()),
        lambda: cache.append(k.cpu(), k.cpu(), pos),
        lambda: cache.append(normal(g, 2, 3, 64, 2).transpose(2, 3), k, pos),
        lambda: cache.append(normal(g, 2, 3, 2, 68)[..., :64], k, pos),
        lambda: cache.append(normal(g, 2, 3 * 2 * 64 + 8)[:, 1:385].view(2, 3, 2, 64), k, pos),
        lambda: cache.attention(q[:1], pos),
        lambda: cache.attention(q.half(), pos),
        lambda: cache.attention(q, pos[:, :2].contiguous()),
        lambda: cache.attention(q[:, :, :3], pos),
        lambda: cache.attention(q, pos, scale=0.0),
        lambda: cache.attention(q, pos, scale=math.nan),
        lambda: cache.attention(q, pos, max_len=0),
        lambda: cache.attention(q, pos, max_len=binding.SD_KV_MAX_LEN + 1),
        lambda: cache.attention(q, pos, out=torch.empty_like(q, dtype=torch.float32)),
        lambda: cache.attention(q, pos, lse=torch.empty(2, 3, 4, device="cuda", dtype=torch.float64)),
        lambda: cache.attention(q, pos, scratch=torch.zeros(1024, dtype=torch.uint8, device="cuda")),
    ]
    before = cache.pool.clone()
    for i, call in enumerate(bad):
        with pytest.raises(binding.SdError):
            call()
            pytest.fail(f"call {i} was not refused")
    assert torch.equal(cache.pool, before)
    with pytest.raises(binding.SdError) as e:
        cache.attention(q, pos, max_len=0)
    assert e.value.status == binding.SD_ERANGE or "max_len" in str(e.value)
