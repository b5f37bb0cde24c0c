"""The rotation and the paged cache on the GPU, through the binding, against plain 64-bit forms."""
import ctypes
import math

import pytest
import torch

from paper_2410_23079_b200 import BuzzError, BuzzPaged, norm_rope
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, E4M3, I8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.int8
KINDS = [(BF16, BF16), (BF16, E4M3), (BF16, I8), (F32, F32), (F32, E4M3), (F32, I8)]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def within(got, want, bound, what=""):
    got, bound = got.double().cpu(), bound.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].nan_to_num(7.0), want[~fine].nan_to_num(7.0)), what
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0.0, (what, float(over.max()), float((got - want)[fine].abs().max()))


# ---- rotation ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,rotary", [(128, 128), (128, 48), (64, 64), (64, 16), (128, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads", [(1, (8, 2)), (17, (7, 1)), (2500, (4, 4))])
def test_norm_rope(cuda_device, dtype, d, rotary, interleaved, tokens, heads):
    g = gen(tokens + d + rotary)
    wide = torch.randn(tokens, sum(heads) + 1, d, generator=g).to(dtype)           # a projection's output with one more head
    q, k = wide[:, :heads[0]], wide[:, heads[0]:sum(heads)]
    pos = torch.randint(-5, 1 << 20, (tokens,), generator=g).to(torch.int32)
    pos[0] = 0 if tokens == 1 else (1 << 31) - 1
    freq = (500000.0 ** (-torch.arange(0, rotary, 2).double() / rotary)).float()
    qw, kw = [(1 + torch.randn(d, generator=g) / 4).to(dtype) for _ in range(2)]
    wd = wide.to(DEV)
    for a, b in ((qw, kw), (None, kw), (None, None)):
        on = lambda x: None if x is None else x.to(DEV)
        qo, ko = norm_rope(wd[:, :heads[0]], wd[:, heads[0]:sum(heads)], pos.to(DEV), freq.to(DEV), on(a), on(b), eps=1e-5, interleaved=interleaved)
        for got, x, w in ((qo, q, a), (ko, k, b)):
            want, bound = ref.norm_rope(x, w, pos, freq, 1e-5, interleaved)
            within(got, want, bound)
    assert torch.equal(wd.cpu(), wide)


def test_norm_rope_in_place_strided_outputs_and_streams(cuda_device):
    g = gen(5)
    wide = torch.randn(33, 13, 128, generator=g).to(BF16)
    pos, freq = torch.arange(33, dtype=torch.int32), (1e4 ** (-torch.arange(0, 128, 2).double() / 128)).float()
    w = torch.ones(128).to(BF16)
    a = wide.to(DEV)
    qo, ko = norm_rope(a[:, :8], a[:, 8:10], pos.to(DEV), freq.to(DEV), w.to(DEV), None)
    b, p, f, ww = wide.to(DEV), pos.to(DEV), freq.to(DEV), w.to(DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    r = norm_rope(b[:, :8], b[:, 8:10], p, f, ww, None, q_out=b[:, :8], k_out=b[:, 8:10], stream=side)
    side.synchronize()
    assert r[0].data_ptr() == b.data_ptr()
    assert torch.equal(b[:, :8], qo) and torch.equal(b[:, 8:10], ko) and torch.equal(b[:, 10:].cpu(), wide[:, 10:])
    empty = norm_rope(a[:0, :8], a[:0, 8:10], p[:0], f)
    assert empty[0].shape == (0, 8, 128)


def test_norm_rope_refusals(cuda_device):
    q, p, f = torch.zeros(4, 2, 64, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV), torch.ones(16, device=DEV)
    for call in (lambda: norm_rope(q, q, p.long(), f), lambda: norm_rope(q, q.bfloat16(), p, f), lambda: norm_rope(q, q, p[:3], f),
                 lambda: norm_rope(q, q, p, f.double()), lambda: norm_rope(q, q[:3], p, f), lambda: norm_rope(q.half(), q.half(), p, f),
                 lambda: norm_rope(q.transpose(0, 1), q, p, f), lambda: norm_rope(q, q, p, f, q_weight=f),
                 lambda: norm_rope(q, q, p, f, q_out=q[:3]), lambda: norm_rope(q, q, p.cpu(), f)):
        with pytest.raises(ValueError):
            call()
    for bad in (f[:4], torch.ones(40, device=DEV)):
        with pytest.raises(BuzzError):
            norm_rope(q, q, p, bad)
    with pytest.raises(BuzzError):
        norm_rope(q, q, p, f, eps=-1.0)
    w = torch.ones(64, device=DEV, requires_grad=True)
    with pytest.raises(ValueError):
        norm_rope(q, q, p, f, q_weight=w)
    with pytest.raises(ValueError):
        norm_rope(q, q, p, f, k_weight=w)
    with torch.no_grad():
        norm_rope(q, q, p, f, q_weight=w)


def test_norm_rope_of_one_token_whatever_its_stride(cuda_device):
    """A single token's rows have no distance that could be wrong."""
    x = torch.randn(3, 5, 64, generator=gen(9)).to(BF16).to(DEV)
    one = x.as_strided((1, 4, 64), (259, 64, 1))
    p, f = torch.tensor([77], dtype=torch.int32, device=DEV), torch.ones(16, device=DEV)
    got, want = norm_rope(one, one, p, f), norm_rope(x[:1, :4], x[:1, :4], p, f)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- pool helpers --------------------------------------------------------------------------------

def poison(pool):
    """Fills every part of a pool with what must never show."""
    for n in ("k", "v", "k_scale", "v_scale", "bounds"):
        t = getattr(pool, n)
        if t is not None:
            if t.dtype in (E4M3, I8):
                t.view(torch.int8).fill_(0x7f)                                   # NaN in e4m3
            else:
                t.fill_(math.nan)


def make(dtype, kind, lens, page, Hq, H, d, g, bounds=True, spare=3, logn=False):
    counts = [-(-n // page) for n in lens]
    pool = BuzzPaged(layers=2, pages=sum(counts) + spare, page_tokens=page, q_heads=Hq, kv_heads=H, head_dim=d, dtype=dtype, cache_dtype=kind,
                     bounds=bounds, logn=logn, device=DEV)
    poison(pool)
    perm = torch.randperm(pool.pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(max(counts), 1) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = perm[at:at + n]
        at += n
    return pool, table, perm[at:]


def pack(rows, H, d):
    return torch.cat(rows) if rows else torch.zeros(0, H, d)


def cu_of(counts):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32)


def kept(x, kind):
    codes, scale = ref.quantise(x, kind)
    return codes if scale is None else codes * scale[..., None]


def dev_lens(lens):
    return torch.tensor(lens, dtype=torch.int32, device=DEV)


# ---- rows in and out -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d,page,H", [(128, 16, 2), (64, 32, 3), (64, 128, 1)])
def test_append_and_read(cuda_device, dtype, kind, d, page, H):
    g = gen(d + page)
    final = [1, page, page + 1, 3 * page - 1, 40, 0, 2 * page + 7]
    pool, table, unused = make(dtype, kind, final, page, H, H, d, g)
    bits = lambda x: x.view(torch.int32 if x.dtype == F32 else torch.uint8).cpu().clone()          # NaN compares by its bits
    before = {n: bits(getattr(pool, n)) for n in ("k", "v", "k_scale", "bounds") if getattr(pool, n) is not None}
    rows = [(torch.randn(n, H, d, generator=g) * torch.exp(2 * torch.randn(n, H, 1, generator=g))).to(dtype) for n in final]
    vals = [torch.randn(n, H, d, generator=g).to(dtype) for n in final]
    rows[3][1, 0] = 0
    rows[3][2, 0, 5] = -3e38
    # in three calls: part of each prompt, the rest but one (now and then nothing), single tokens
    at = [0] * len(final)
    for cut in (lambda n: n // 2, lambda n: n - 1, lambda n: n):
        upto = [max(a, cut(n)) for a, n in zip(at, final)]
        new = [u - a for u, a in zip(upto, at)]
        k = pack([r[a:u] for r, a, u in zip(rows, at, upto)], H, d).to(DEV)
        v = pack([r[a:u] for r, a, u in zip(vals, at, upto)], H, d).to(DEV)
        if k.shape[0]:
            pool.append(1, k, v, dev_lens(upto), table.to(DEV), cu_of(new).to(DEV), max(new))
        at = upto
    assert pool.status() == 0
    ko, vo = torch.full((sum(final), H, d), 9.0, dtype=dtype, device=DEV), torch.full((sum(final), H, d), 9.0, dtype=dtype, device=DEV)
    pool.read(1, dev_lens(final), table.to(DEV), ko, vo, cu_of(final).to(DEV))
    assert pool.status() == 0
    for got, x in ((ko, rows), (vo, vals)):
        assert torch.equal(got.cpu(), kept(pack(x, H, d), kind).to(dtype)), "rows read back"
    for b, n in enumerate(final):
        want = ref.page_bounds(rows[b], page)
        for i in range(-(-n // page)):
            assert torch.equal(pool.bounds[1, table[b, i]].double().cpu(), want[i]), (b, i)
    # slots behind a sequence, pages of nobody and the other layer are as they were
    for n, old in before.items():
        new = bits(getattr(pool, n))
        assert torch.equal(new[0], old[0]), n
        assert torch.equal(new[1][unused.long()], old[1][unused.long()]), n
        if n != "bounds":
            for b, m in enumerate(final):
                if m % page:
                    p = int(table[b, m // page])
                    assert torch.equal(new[1][p][:, m % page:], old[1][p][:, m % page:]), (n, b)


@pytest.mark.parametrize("dtype,kind", KINDS)
def test_append_one_token_each_without_cu_seqlens(cuda_device, dtype, kind):
    g = gen(1)
    page, H, d, lens = 16, 5, 64, [1, 16, 17, 33]
    pool, table, _ = make(dtype, kind, lens, page, H, H, d, g)
    k, v = torch.randn(4, H, d, generator=g).to(dtype), torch.randn(4, H, d, generator=g).to(dtype)
    pool.bounds.zero_()
    pool.append(0, k.to(DEV), v.to(DEV), dev_lens(lens), table.to(DEV))
    ko, vo = torch.empty_like(k, device=DEV), torch.empty_like(v, device=DEV)
    pool.read(0, dev_lens(lens), table.to(DEV), ko, vo)
    assert pool.status() == 0
    assert torch.equal(ko.cpu(), kept(k, kind).to(dtype)) and torch.equal(vo.cpu(), kept(v, kind).to(dtype))
    for b, n in enumerate(lens):                             # slot 0 begins a page's bounds, a later one widens them
        got = pool.bounds[0, table[b, (n - 1) // page]].cpu()
        x = k[b]
        want = torch.stack([x, x], 1) if (n - 1) % page == 0 else torch.stack([x.clamp_max(0), x.clamp_min(0)], 1)
        assert torch.equal(got.float(), want.float()), b


@pytest.mark.parametrize("dtype,kind", [(BF16, E4M3), (F32, I8), (BF16, BF16)])
def test_rows_with_infinities_and_nan(cuda_device, dtype, kind):
    pool, table, _ = make(dtype, kind, [16], 16, 1, 1, 64, gen(2))
    k = torch.randn(16, 1, 64, generator=gen(3)).to(dtype)
    k[3, 0, 7], k[5, 0, 9], k[6, 0, 1] = math.inf, math.nan, -math.inf
    pool.append(0, k.to(DEV), k.to(DEV), dev_lens([16]), table.to(DEV), cu_of([16]).to(DEV))
    ko, vo = torch.empty_like(k, device=DEV), torch.empty_like(k, device=DEV)
    pool.read(0, dev_lens([16]), table.to(DEV), ko, vo, cu_of([16]).to(DEV))
    got = ko.cpu()
    if kind == dtype:
        assert torch.equal(got.nan_to_num(nan=1234.0), k.nan_to_num(nan=1234.0))
    else:
        for r in range(16):
            assert bool(got[r].isnan().all()) == (r in (3, 5, 6)), r
    assert torch.equal(pool.bounds[0, table[0, 0]].double().cpu(), ref.page_bounds(k, 16)[0])


@pytest.mark.parametrize("kind,top", [(E4M3, 448.0), (I8, 127.0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("factor", [1.0, 2.0 ** -90, 3.0, 1.7e30, 0.1])
def test_codes_at_their_borders(cuda_device, kind, top, dtype, factor):
    """Values on the borders between codes and one, two and three units beside them, at scales that are and are not powers of two."""
    if kind == I8:
        mids = torch.arange(127).double() + 0.5
    else:
        grid = torch.cat([torch.arange(0, 9).double() * 2.0 ** -9] + [torch.arange(8, 16).double() * 2.0 ** e for e in range(-9, 6)]).unique()
        grid = grid[grid <= 448]
        mids = (grid[1:] + grid[:-1]) / 2
    rows = []
    for shift in range(-3, 4):
        x = (mids * factor).to(dtype)
        bits = x.view(torch.int16 if dtype == BF16 else torch.int32)
        rows.append((bits + shift).view(dtype) * torch.where(torch.arange(len(mids)) % 2 == 0, 1.0, -1.0).to(dtype))
    x = torch.cat(rows)
    n = -(-x.numel() // 63)
    k = torch.zeros(n, 1, 64, dtype=dtype)
    k.view(n, 64)[:, :63] = torch.cat([x, torch.zeros(63 * n - x.numel(), dtype=dtype)]).view(n, 63)
    k[:, 0, 63] = top * factor
    pool, table, _ = make(dtype, kind, [n], 16, 1, 1, 64, gen(1), bounds=False)
    pool.append(0, k.to(DEV), k.to(DEV), dev_lens([n]), table.to(DEV), cu_of([n]).to(DEV))
    assert pool.status() == 0
    codes, scale = ref.quantise(k, kind)
    at = torch.arange(n)
    got = pool.k[0].view(torch.int8).cpu().view(pool.pages, 16, 64)[table[0, at // 16].long(), at % 16].view(kind).double()
    assert torch.equal(got, codes[:, 0])
    assert torch.equal(pool.k_scale[0].cpu().view(pool.pages, 16)[table[0, at // 16].long(), at % 16].double(), scale[:, 0])


# ---- attention -----------------------------------------------------------------------------------

def attend_case(dtype, kind, lens, page, Hq, H, d, seed, logn=False, max_len=None):
    g = gen(seed)
    pool, table, _ = make(dtype, kind, lens, page, Hq, H, d, g, logn=logn)
    ks = [torch.randn(n, H, d, generator=g).to(dtype) * torch.where(torch.rand(n, H, 1, generator=g) < 0.05, 4.0, 1.0).to(dtype) for n in lens]
    vs = [torch.randn(n, H, d, generator=g).to(dtype) for n in lens]
    if sum(lens):
        pool.append(1, pack(ks, H, d).to(DEV), pack(vs, H, d).to(DEV), dev_lens(lens), table.to(DEV), cu_of(lens).to(DEV), max(lens))
    q = torch.randn(len(lens), Hq, d, generator=g).to(dtype)
    out, lse = torch.full((len(lens), Hq, d), 77.0, dtype=dtype, device=DEV), torch.full((len(lens), Hq), 77.0, device=DEV)
    pool.decode(1, q.to(DEV), dev_lens(lens), table.to(DEV), max(lens) if max_len is None else max_len, out, lse=lse)
    assert pool.status() == 0
    for b, n in enumerate(lens):
        scale = d ** -0.5 * (math.log(max(n, 1)) / math.log(512) if logn else 1.0)
        o, e, ob, eb = ref.attention(q[b], kept(ks[b], kind).transpose(0, 1), kept(vs[b], kind).transpose(0, 1), dtype, scale, kind)
        within(out[b], o, ob, ("out", b, n))
        within(lse[b], e, eb, ("lse", b, n))
    return pool, table, ks, vs, q, out


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,H,page", [(2, 2, 16), (8, 1, 32), (6, 3, 64), (8, 2, 128)])
def test_decode_lengths(cuda_device, dtype, kind, d, Hq, H, page):
    attend_case(dtype, kind, [1, 0, 15, 16, 17, 63, 64, 65, 127, 128, 129, 0, 300, 511, 1000], page, Hq, H, d, 7 * d + Hq + page)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("Hq,H,lens", [(1, 1, [9001]), (32, 8, [517]), (8, 8, [2049, 3, 4095]), (4, 2, [0]), (16, 2, [1])])
def test_decode_split_over_the_length(cuda_device, dtype, kind, Hq, H, lens):
    attend_case(dtype, kind, lens, 16, Hq, H, 128, 11 + Hq)


def test_decode_more_sequences_than_threads(cuda_device):
    lens = [(37 * i) % 150 for i in range(700)]
    attend_case(BF16, I8, lens, 32, 2, 1, 64, 3)


@pytest.mark.parametrize("dtype,kind", [(BF16, BF16), (F32, E4M3)])
def test_decode_logn(cuda_device, dtype, kind):
    attend_case(dtype, kind, [1, 2, 100, 512, 1500], 32, 4, 2, 128, 5, logn=True)


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("lens", [[1024, 1, 0, 1000], [700, 2100], [1500] * 19])
def test_decode_one_block_per_head_or_split(cuda_device, dtype, kind, lens):
    """Lengths around the limit up to which a block does a (sequence, KV head) alone, and more heads than SMs."""
    attend_case(dtype, kind, lens, 64, 16, 8, 128, len(lens))


def test_decode_is_reproducible_and_ignores_a_loose_bound(cuda_device):
    pool, table, ks, vs, q, out = attend_case(BF16, BF16, [3000, 17, 1], 16, 8, 2, 128, 9)
    for _ in range(5):
        again = torch.empty_like(out)
        pool.decode(1, q.to(DEV), dev_lens([3000, 17, 1]), table.to(DEV), 3000, again)
        assert torch.equal(again, out)
    again.fill_(3.0)
    pool.decode(1, q.to(DEV), dev_lens([3000, 17, 1]), table.to(DEV), table.shape[1] * 16, again)
    assert torch.equal(again, out)


def test_decode_logits_of_minus_infinity_and_extreme_scales(cuda_device):
    """Keys whose logits overflow to -inf weigh nothing; a query against huge keys takes the largest alone."""
    g = gen(21)
    pool, table, _ = make(BF16, BF16, [40], 16, 1, 1, 64, g)
    q = torch.ones(1, 1, 64, dtype=BF16)
    k, v = torch.randn(40, 1, 64, generator=g).to(BF16), torch.randn(40, 1, 64, generator=g).to(BF16)
    k[:16] = -3e38                                            # a whole tile, and more, of -inf
    k[20] = -3e38
    pool.append(0, k.to(DEV), v.to(DEV), dev_lens([40]), table.to(DEV), cu_of([40]).to(DEV))
    out, lse = torch.empty(1, 1, 64, dtype=BF16, device=DEV), torch.empty(1, 1, device=DEV)
    pool.decode(0, q.to(DEV), dev_lens([40]), table.to(DEV), 40, out, lse=lse)
    keep = [i for i in range(16, 40) if i != 20]
    o, e, ob, eb = ref.attention(q[0], k[keep].double().transpose(0, 1), v[keep].double().transpose(0, 1), BF16)
    within(out[0], o, ob)
    within(lse[0], e, eb)
    pool.decode(0, q.to(DEV), dev_lens([16]), table.to(DEV), 16, out, lse=lse)       # nothing else: a row of nothing
    assert torch.equal(out.cpu(), torch.zeros(1, 1, 64, dtype=BF16)) and float(lse) == -math.inf


@pytest.mark.parametrize("dtype,kind", KINDS)
@pytest.mark.parametrize("H,lens", [(1, [1100]), (2, [9000]), (8, [1100] * 20)])
def test_decode_does_not_lose_a_nan(cuda_device, dtype, kind, H, lens):
    """Keys that are NaN, a tile or a block's whole share of them: the output of their sequence and head is NaN, the
    others are as without them. A cluster per head, the line, more heads than SMs."""
    g = gen(22)
    pool, table, _ = make(dtype, kind, lens, 16, H, H, 128, g)
    k, v = [torch.randn(sum(lens), H, 128, generator=g).to(dtype).to(DEV) for _ in range(2)]
    q = torch.randn(len(lens), H, 128, generator=g).to(dtype).to(DEV)
    t = table.to(DEV)
    pool.append(0, k, v, dev_lens(lens), t, cu_of(lens).to(DEV), max(lens))
    good, out = torch.empty_like(q), torch.empty_like(q)
    pool.decode(0, q, dev_lens(lens), t, max(lens), good)
    assert bool(good.isfinite().all())
    for lo, hi in ((0, lens[0]), (0, 160), (384, 800), (lens[0] - 1, lens[0])):
        bad = k.clone()
        bad[lo:hi, 0] = math.nan
        pool.append(0, bad, v, dev_lens(lens), t, cu_of(lens).to(DEV), max(lens))
        lse = torch.zeros(len(lens), H, device=DEV)
        pool.decode(0, q, dev_lens(lens), t, max(lens), out, lse=lse)
        assert bool(out[0, 0].isnan().all()) and bool(lse[0, 0].isnan()), (lo, hi)
        out[0, 0] = good[0, 0]
        assert torch.equal(out, good), (lo, hi)
    assert pool.status() == 0


def test_decode_bad_lengths_and_pages(cuda_device):
    g = gen(31)
    lens = [100, 50, 70]
    pool, table, ks, vs, q, out = attend_case(BF16, E4M3, lens, 16, 2, 1, 64, 31)
    good = out.clone()
    for bad in (-1, 101, 1 << 30):
        out.fill_(5.0)
        lse = torch.full((3, 2), 5.0, device=DEV)
        pool.decode(1, q.to(DEV), dev_lens([100, bad, 70]), table.to(DEV), 100, out, lse=lse)
        assert pool.status() == -1 and pool.status() == 0
        assert torch.equal(out[[0, 2]], good[[0, 2]]) and bool((out[1] == 5.0).all()) and bool((lse[1] == 5.0).all())
    for page in (-1, pool.pages, 1 << 30):
        t = table.clone()
        t[2, 1] = page                                        # tokens 16..31 of the last sequence take no part
        pool.decode(1, q.to(DEV), dev_lens(lens), t.to(DEV), 100, out)
        assert pool.status() == -1
        assert torch.equal(out[:2], good[:2])
        keep = [i for i in range(70) if not 16 <= i < 32]
        o, _, ob, _ = ref.attention(q[2], kept(ks[2][keep], E4M3).transpose(0, 1), kept(vs[2][keep], E4M3).transpose(0, 1), BF16, kind=E4M3)
        within(out[2], o, ob)


def test_append_bad_arguments_on_the_device(cuda_device):
    pool, table, _ = make(BF16, BF16, [40, 40], 16, 1, 1, 64, gen(41))
    keep = pool.k.view(torch.int16).clone()
    x = torch.ones(8, 1, 64, dtype=BF16, device=DEV)
    t = table.to(DEV)
    for lens, cu in (([3, 4], [0, 4, 8]), ([65, 1000], [0, 4, 8]), ([-1, 8], [0, 0, 8]), ([20, 20], [0, 9, 8]), ([20, 20], [0, 0, 9])):
        pool.append(0, x, x, dev_lens(lens), t, torch.tensor(cu, dtype=torch.int32, device=DEV), 8)
        assert pool.status() == -1, (lens, cu)
    t2 = t.clone()
    t2[0, 0], t2[1, 0] = -1, pool.pages
    keep2 = pool.k.view(torch.int16).clone()
    pool.append(0, x, x, dev_lens([4, 4]), t2, torch.tensor([0, 4, 8], dtype=torch.int32, device=DEV), 4)
    assert pool.status() == -1
    assert torch.equal(pool.k.view(torch.int16), keep2)
    assert not torch.equal(keep, keep2)                       # the sound sequences of the calls above were written


def test_offsets_beyond_32_bits(cuda_device):
    """Pages whose rows lie beyond 2^31 elements and 2^32 bytes of the pool."""
    H, page, d = 8, 128, 128
    pool = BuzzPaged(layers=1, pages=20000, page_tokens=page, q_heads=8, kv_heads=H, head_dim=d, dtype=BF16, bounds=True, device=DEV)
    g = gen(51)
    lens = [300, 129]
    table = torch.tensor([[19999, 3, 17001], [16500, 19998, -1]], dtype=torch.int32)
    ks, vs = [[torch.randn(n, H, d, generator=g).to(BF16) for n in lens] for _ in range(2)]
    pool.append(0, pack(ks, H, d).to(DEV), pack(vs, H, d).to(DEV), dev_lens(lens), table.to(DEV), cu_of(lens).to(DEV))
    ko, vo = torch.empty(429, H, d, dtype=BF16, device=DEV), torch.empty(429, H, d, dtype=BF16, device=DEV)
    pool.read(0, dev_lens(lens), table.to(DEV), ko, vo, cu_of(lens).to(DEV))
    assert torch.equal(ko.cpu(), pack(ks, H, d)) and torch.equal(vo.cpu(), pack(vs, H, d))
    q, out = torch.randn(2, 8, d, generator=g).to(BF16), torch.empty(2, 8, d, dtype=BF16, device=DEV)
    pool.decode(0, q.to(DEV), dev_lens(lens), table.to(DEV), 384, out)
    for b in range(2):
        o, _, ob, _ = ref.attention(q[b], ks[b].double().transpose(0, 1), vs[b].double().transpose(0, 1), BF16)
        within(out[b], o, ob)
    sel = torch.empty(2, H, 2, dtype=torch.int32, device=DEV)
    pool.select(0, q.to(DEV), dev_lens(lens), table.to(DEV), 384, 0, 1, 1, sel)
    for b in range(2):
        want = ref.choose(q[b], ref.page_bounds(ks[b], page), 0, 1, 1)
        assert sel[b].tolist() == [w + [-1] * (2 - len(w)) for w in want]
    assert pool.status() == 0


# ---- choice of pages, and attention over them ----------------------------------------------------

def select_case(dtype, kind, lens, page, Hq, H, d, sink, recent, top, seed, tie=False):
    g = gen(seed)
    pool, table, _ = make(dtype, kind, lens, page, Hq, H, d, g)
    ks = [torch.randn(n, H, d, generator=g).to(dtype) for n in lens]
    if tie:                                                   # few different pages: many equal scores
        for x in ks:
            for i in range(0, x.shape[0] - page + 1, page):
                x[i:i + page] = x[:page] * (1 + (i // page) % 3)
    vs = [torch.randn(n, H, d, generator=g).to(dtype) for n in lens]
    pool.append(1, pack(ks, H, d).to(DEV), pack(vs, H, d).to(DEV), dev_lens(lens), table.to(DEV), cu_of(lens).to(DEV), max(lens))
    q = torch.randn(len(lens), Hq, d, generator=g).to(dtype)
    n = sink + recent + top
    sel = torch.full((len(lens), H, n), 99, dtype=torch.int32, device=DEV)
    out, lse = torch.empty(len(lens), Hq, d, dtype=dtype, device=DEV), torch.empty(len(lens), Hq, device=DEV)
    pool.select(1, q.to(DEV), dev_lens(lens), table.to(DEV), max(lens), sink, recent, top, sel)
    pool.decode(1, q.to(DEV), dev_lens(lens), table.to(DEV), max(lens), out, lse=lse, selected=sel)
    assert pool.status() == 0
    G = Hq // H
    for b, m in enumerate(lens):
        want = ref.choose(q[b], ref.page_bounds(ks[b], page), sink, recent, top)
        assert sel[b].tolist() == [w + [-1] * (n - len(w)) for w in want], b
        k, v = kept(ks[b], kind).transpose(0, 1), kept(vs[b], kind).transpose(0, 1)
        for h in range(H):
            rows = [i for p in want[h] for i in range(p * page, min(m, (p + 1) * page))]
            o, e, ob, eb = ref.attention(q[b, h * G:(h + 1) * G], k[h:h + 1, rows], v[h:h + 1, rows], dtype, kind=kind)
            within(out[b, h * G:(h + 1) * G], o, ob, (b, h))
            within(lse[b, h * G:(h + 1) * G], e, eb, (b, h))


@pytest.mark.parametrize("dtype,kind,d", [(BF16, BF16, 128), (BF16, E4M3, 64), (F32, F32, 64), (F32, I8, 128)])
@pytest.mark.parametrize("Hq,H,page,sink,recent,top", [(2, 2, 16, 1, 2, 5), (8, 1, 32, 0, 1, 3), (8, 2, 16, 3, 1, 0), (3, 3, 64, 0, 3, 1)])
def test_select_and_decode(cuda_device, dtype, kind, d, Hq, H, page, sink, recent, top):
    select_case(dtype, kind, [1, 0, 16, 100, 401, 1000, 1025], page, Hq, H, d, sink, recent, top, d + Hq + page)


@pytest.mark.parametrize("top", [1, 7, 200, 1500])
def test_select_many_pages(cuda_device, top):
    select_case(BF16, BF16, [40000, 12345], 16, 2, 1, 64, 2, 4, top, top)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_select_ties_go_to_the_lowest_page(cuda_device, dtype):
    select_case(dtype, dtype, [1600, 800, 2000], 16, 2, 2, 64, 1, 1, 11, 13, tie=True)


@pytest.mark.parametrize("pages,heads", [(500, 1), (900, 1), (9000, 2)])
def test_select_many_equal_scores(cuda_device, pages, heads):
    """A crowd at the border that is one value: the lowest of its pages are kept."""
    n = 16 * pages
    pool, table, _ = make(BF16, BF16, [n], 16, heads, heads, 64, gen(7))
    b = torch.zeros(pages, heads, 2, 64, dtype=BF16)
    b[100, :, 1, 0], b[pages - 7, :, 1, 0], b[3, :, 0, 0], b[3, :, 1, 0] = 1.0, 2.0, -1.0, -0.5
    pool.bounds[0, table[0, :pages].long()] = b.to(DEV)
    q = torch.zeros(1, heads, 64, dtype=BF16)
    q[..., 0] = 1.0
    for top in (1, 2, 3, 40, 300):
        sel = torch.empty(1, heads, top + 2, dtype=torch.int32, device=DEV)
        pool.select(0, q.to(DEV), dev_lens([n]), table.to(DEV), n, 1, 1, top, sel)
        order = [pages - 7, 100] + [i for i in range(1, pages - 1) if i not in (3, 100, pages - 7)] + [3]
        assert sel[0].tolist() == [[0] + sorted(order[:top]) + [pages - 1]] * heads, top
    assert pool.status() == 0


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F32, 128), (BF16, 64)])
def test_select_with_many_heads(cuda_device, dtype, d):
    select_case(dtype, dtype, [11000, 3, 9999, 400, 700], 16, 32, 32, d, 1, 3, 50, d)


def test_select_special_scores(cuda_device):
    """Zeros of both signs tie, infinities and NaN have their places."""
    pool, table, _ = make(F32, F32, [160], 16, 1, 1, 64, gen(1))
    b = torch.zeros(10, 1, 2, 64)
    b[1, 0, :, 0] = -0.0
    b[2, 0, :, 0], b[3, 0, :, 0], b[4, 0, :, 0] = -1.0, math.inf, -math.inf
    b[6, 0, 0, 0], b[6, 0, 1, 1] = math.nan, math.nan
    b[7, 0, :, 0] = 2.0
    pool.bounds[0, table[0, :10].long()] = b.to(DEV)
    q = torch.zeros(1, 1, 64)
    q[0, 0, 0] = 1.0
    for top in range(0, 9):
        sel = torch.empty(1, 1, top + 1, dtype=torch.int32, device=DEV)
        pool.select(0, q.to(DEV), dev_lens([160]), table.to(DEV), 160, 0, 1, top, sel)
        order = [6, 3, 7, 0, 1, 5, 8, 2, 4]                   # NaN (a NaN bound), infinity, 2, zeros, -1, -infinity
        assert sel[0, 0].tolist() == sorted(order[:top]) + [9], top


@pytest.mark.parametrize("dtype,d,H,group", [(BF16, 128, 2, 4), (BF16, 64, 1, 1), (F32, 64, 3, 2), (F32, 128, 1, 8)])
@pytest.mark.parametrize("pages", [60, 700])
def test_select_with_infinite_and_nan_keys(cuda_device, dtype, d, H, group, pages):
    """Keys that hold infinities and NaN, whole pages of NaN, and queries that do and do not reach them."""
    g = gen(pages + d)
    pool, table, _ = make(dtype, dtype, [16 * pages], 16, H * group, H, d, g)
    k = torch.randn(pages, 16, H, d, generator=g).to(dtype)
    for i in range(0, pages, 3):
        k[i, int(torch.randint(16, (1,), generator=g)), :, int(torch.randint(d, (1,), generator=g))] = (math.inf, -math.inf, math.nan)[i // 3 % 3]
    k[7, :, :, 3], k[8] = math.nan, math.nan
    k = k.view(-1, H, d)
    pool.append(0, k.to(DEV), k.to(DEV), dev_lens([16 * pages]), table.to(DEV), cu_of([16 * pages]).to(DEV))
    bounds = ref.page_bounds(k, 16)
    q = torch.randn(1, H * group, d, generator=g)
    for q in (q, q.abs(), -q.abs(), q * (torch.rand(1, H * group, d, generator=g) < 0.5)):
        q = q.to(dtype)
        for top in (1, 4, 15, 40):
            sel = torch.empty(1, H, top + 2, dtype=torch.int32, device=DEV)
            pool.select(0, q.to(DEV), dev_lens([16 * pages]), table.to(DEV), 16 * pages, 1, 1, top, sel)
            assert sel[0].tolist() == ref.choose(q[0], bounds, 1, 1, top), top
    assert pool.status() == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bounds_and_scores_of_subnormal_keys(cuda_device, dtype):
    g = gen(77)
    pool, table, _ = make(dtype, dtype, [1600], 16, 2, 1, 64, g)
    k = (torch.randn(1600, 1, 64, generator=g).double() * 2.0 ** -130).to(dtype)
    pool.append(0, k.to(DEV), k.to(DEV), dev_lens([1600]), table.to(DEV), cu_of([1600]).to(DEV))
    bounds = ref.page_bounds(k, 16)
    assert float(bounds.abs().max()) > 0
    assert torch.equal(pool.bounds[0, table[0, :100].long()].double().cpu(), bounds)
    for scale in (1.0, 2.0 ** -130):
        q = (torch.randn(1, 2, 64, generator=g).double() * scale).to(dtype)
        sel = torch.empty(1, 1, 12, dtype=torch.int32, device=DEV)
        pool.select(0, q.to(DEV), dev_lens([1600]), table.to(DEV), 1600, 1, 1, 10, sel)
        assert sel[0].tolist() == ref.choose(q[0], bounds, 1, 1, 10)


def test_select_bad_lengths_and_pages(cuda_device):
    g = gen(61)
    lens = [320, 320]
    pool, table, _ = make(BF16, BF16, lens, 16, 1, 1, 64, g)
    k = torch.randn(640, 1, 64, generator=g).to(BF16).to(DEV)
    pool.append(0, k, k, dev_lens(lens), table.to(DEV), cu_of(lens).to(DEV))
    q = torch.randn(2, 1, 64, generator=g).to(BF16).to(DEV)
    good = torch.empty(2, 1, 6, dtype=torch.int32, device=DEV)
    pool.select(0, q, dev_lens(lens), table.to(DEV), 320, 1, 1, 4, good)
    sel = torch.full_like(good, 55)
    pool.select(0, q, dev_lens([321, 320]), table.to(DEV), 320, 1, 1, 4, sel)
    assert pool.status() == -1
    assert bool((sel[0] == 55).all()) and torch.equal(sel[1], good[1])
    t = table.clone()
    t[0, 7] = -5
    pool.select(0, q, dev_lens(lens), t.to(DEV), 320, 1, 1, 18, torch.empty(2, 1, 20, dtype=torch.int32, device=DEV))
    assert pool.status() == 0                                 # every page is kept: none is scored
    sel18 = torch.empty(2, 1, 19, dtype=torch.int32, device=DEV)
    pool.select(0, q, dev_lens(lens), t.to(DEV), 320, 1, 1, 17, sel18)
    assert pool.status() == -1
    assert sel18[0, 0].tolist() == [i for i in range(20) if i != 7]      # the bad page is below all others
    # a choice that names pages outside its sequence: their tokens take no part
    out = torch.empty(2, 1, 64, dtype=BF16, device=DEV)
    want = torch.empty_like(out)
    pool.decode(0, q, dev_lens(lens), table.to(DEV), 320, want, selected=torch.tensor([[[3, 5]], [[3, 5]]], dtype=torch.int32, device=DEV))
    assert pool.status() == 0
    pool.decode(0, q, dev_lens(lens), table.to(DEV), 320, out, selected=torch.tensor([[[3, 5]], [[20, -1]]], dtype=torch.int32, device=DEV))
    assert pool.status() == -1
    assert torch.equal(out[0], want[0]) and bool((out[1] == 0).all())


def test_a_page_listed_twice_counts_twice(cuda_device):
    pool, table, ks, vs, q, out = attend_case(BF16, I8, [60], 16, 2, 1, 64, 65)
    pool.decode(1, q.to(DEV), dev_lens([60]), table.to(DEV), 60, out, selected=torch.tensor([[[3, 1, 1]]], dtype=torch.int32, device=DEV))
    assert pool.status() == 0
    rows = list(range(48, 60)) + list(range(16, 32)) * 2
    o, _, ob, _ = ref.attention(q[0], kept(ks[0][rows], I8).transpose(0, 1), kept(vs[0][rows], I8).transpose(0, 1), BF16, kind=I8)
    within(out[0], o, ob)


@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("kind", [BF16, E4M3])
def test_selection_in_any_order(cuda_device, page, kind):
    """The partly filled last page first and in between: its empty slots take no part wherever it stands."""
    n = 5 * page + 3
    pool, table, ks, vs, q, out = attend_case(BF16, kind, [n], page, 4, 1, 128, 69)
    for order in ([5, 0, 3], [2, 5, 1], [4, 0, 5], [5, 4, 3, 2, 1, 0]):
        sel = torch.tensor([[order]], dtype=torch.int32, device=DEV)
        pool.decode(1, q.to(DEV), dev_lens([n]), table.to(DEV), n, out, selected=sel)
        assert pool.status() == 0
        rows = [i for p in order for i in range(p * page, min(n, (p + 1) * page))]
        o, _, ob, _ = ref.attention(q[0], kept(ks[0][rows], kind).transpose(0, 1), kept(vs[0][rows], kind).transpose(0, 1), BF16, kind=kind)
        within(out[0], o, ob, order)


def test_rows_behind_the_last_sequence(cuda_device):
    """Packed rows that belong to no sequence are neither read nor written."""
    g = gen(66)
    pool, table, _ = make(BF16, E4M3, [20, 5], 16, 2, 2, 64, g)
    x = torch.randn(40, 2, 64, generator=g).to(BF16)
    x[25:] = math.nan
    cu, lens, t = cu_of([20, 5]).to(DEV), dev_lens([20, 5]), table.to(DEV)
    pool.append(0, x.to(DEV), x.to(DEV), lens, t, cu, 20)
    ko, vo = [torch.full((40, 2, 64), 3.0, dtype=BF16, device=DEV) for _ in range(2)]
    pool.read(0, lens, t, ko, vo, cu, 20)
    assert pool.status() == 0
    for y in (ko, vo):
        assert torch.equal(y[:25].cpu(), kept(x[:25], E4M3).to(BF16)) and bool((y[25:] == 3.0).all())


def test_everything_on_a_stream_of_its_own(cuda_device):
    g = gen(67)
    want_pool, table, ks, vs, q, want = attend_case(BF16, E4M3, [900, 30], 16, 4, 2, 64, 68)
    pool, table, _ = make(BF16, E4M3, [900, 30], 16, 4, 2, 64, g)
    k, v, lens, t, cu, qd = pack(ks, 2, 64).to(DEV), pack(vs, 2, 64).to(DEV), dev_lens([900, 30]), table.to(DEV), cu_of([900, 30]).to(DEV), q.to(DEV)
    out, all_pages = torch.empty_like(want), torch.empty_like(want)
    sel = torch.empty(2, 2, 57, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    pool.append(0, k, v, lens, t, cu, 900, stream=side)
    pool.decode(0, qd, lens, t, 900, out, stream=side)
    pool.select(0, qd, lens, t, 900, 1, 1, 55, sel, stream=side)
    pool.decode(0, qd, lens, t, 900, all_pages, selected=sel, stream=side)
    assert pool.status(side) == 0
    assert torch.equal(out, want) and torch.equal(all_pages, want)
    with pytest.raises(ValueError):
        norm_rope(qd.float().requires_grad_(), qd.float(), torch.zeros(2, dtype=torch.int32, device=DEV), torch.ones(8, device=DEV))


# ---- arguments -----------------------------------------------------------------------------------

def test_refusals(cuda_device):
    pool, table, _ = make(BF16, E4M3, [40, 30], 16, 4, 2, 64, gen(71))
    t, lens = table.to(DEV), dev_lens([40, 30])
    q, out = torch.zeros(2, 4, 64, dtype=BF16, device=DEV), torch.zeros(2, 4, 64, dtype=BF16, device=DEV)
    x = torch.zeros(2, 2, 64, dtype=BF16, device=DEV)
    sel = torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV)
    for call in (lambda: pool.decode(0, q.float(), lens, t, 40, out), lambda: pool.decode(0, q[:1], lens, t, 40, out),
                 lambda: pool.decode(0, q, lens.long(), t, 40, out), lambda: pool.decode(0, q, lens, t[:1], 40, out),
                 lambda: pool.decode(0, q, lens, t.cpu(), 40, out), lambda: pool.decode(0, q, lens, t, 40, out.transpose(0, 1)),
                 lambda: pool.decode(0, q, lens, t, 40, out, lse=out[..., 0]), lambda: pool.decode(0, q, lens, t, 40, out, selected=sel[:, :1]),
                 lambda: pool.decode(0, q, lens, t, 40, out, selected=sel[..., :0].contiguous()),
                 lambda: pool.append(0, x, x[:1], lens, t), lambda: pool.append(0, x[:1], x[:1], lens, t),
                 lambda: pool.append(0, x.float(), x.float(), lens, t), lambda: pool.append(0, x, x, lens, t, cu_seqlens=lens),
                 lambda: pool.select(0, q, lens, t, 40, 1, 1, 2, sel), lambda: pool.select(0, q, lens, t, 40, 0, 1, 2, sel.float())):
        with pytest.raises(ValueError):
            call()
    before = pool.launch_count()
    for call in (lambda: pool.decode(2, q, lens, t, 40, out), lambda: pool.decode(-1, q, lens, t, 40, out), lambda: pool.decode(0, q, lens, t, -1, out),
                 lambda: pool.decode(0, q, lens, t, 16 * t.shape[1] + 1, out), lambda: pool.append(9, x, x, lens, t),
                 lambda: pool.append(0, x, x, lens, t, cu_seqlens=cu_of([1, 1]).to(DEV), max_new=3),
                 lambda: pool.append(0, x, x, lens, t, cu_seqlens=cu_of([1, 1]).to(DEV), max_new=0),
                 lambda: pool.select(0, q, lens, t, 40, 3, 0, 0, sel), lambda: pool.select(0, q, lens, t, 40, -1, 1, 3, sel),
                 lambda: pool.select(0, q, lens, t, 40, 0, 4, -1, sel), lambda: pool.select(0, q, lens, t, 4000, 1, 1, 1, sel)):
        with pytest.raises(BuzzError) as e:
            call()
        assert e.value.code == -1
    n = ctypes.c_size_t()
    lib, h = pool._lib, pool._h
    assert lib.buzz_paged_workspace_bytes(h, 0, 1, 0, ctypes.byref(n), ctypes.byref(n)) == -1
    assert lib.buzz_paged_workspace_bytes(h, 1, 1, -1, ctypes.byref(n), ctypes.byref(n)) == -1
    many = torch.zeros(2, 60000, dtype=torch.int32, device=DEV)
    assert lib.buzz_paged_workspace_bytes(h, 2, 960000, 0, ctypes.byref(n), None) == 0 and n.value > 0
    for ws, size in ((None, n.value), (x.data_ptr(), n.value - 1), (x.data_ptr() + 8, n.value)):     # none, too small, misaligned
        assert lib.buzz_paged_decode(h, 0, q.data_ptr(), lens.data_ptr(), many.data_ptr(), 60000, 2, 960000, None, 0, out.data_ptr(), None,
                                     ws, size, None) == -1
    wide = torch.zeros(2, 600, dtype=torch.int32, device=DEV)
    for ws in (None, x.data_ptr()):                           # no workspace, and one that is too small
        assert lib.buzz_paged_select(h, 0, q.data_ptr(), lens.data_ptr(), wide.data_ptr(), 600, 2, 9600, 1, 1, 1, sel.data_ptr(), ws, 8, None) == -1
    assert pool.launch_count() == before
    bare, table, _ = make(BF16, BF16, [40, 30], 16, 4, 2, 64, gen(72), bounds=False)
    with pytest.raises(ValueError):
        bare.select(0, q, lens, t, 40, 1, 1, 1, sel)
    with pytest.raises(ValueError):
        BuzzPaged(layers=1, pages=2, page_tokens=16, q_heads=2, kv_heads=2, head_dim=64, dtype=BF16, buffers={"k": bare.k}, device=DEV)
    with pytest.raises(ValueError):
        BuzzPaged(layers=1, pages=2, page_tokens=16, q_heads=2, kv_heads=2, head_dim=64, dtype=torch.float16, device=DEV)
    with pytest.raises(BuzzError):
        BuzzPaged(layers=1, pages=2, page_tokens=24, q_heads=2, kv_heads=2, head_dim=64, dtype=BF16, device=DEV)


# ---- a run of them together ----------------------------------------------------------------------

@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("captured", [False, True])
def test_prompts_then_steps_of_one_layer(cuda_device, kind, captured):
    """Projections -> norm_rope -> append -> (select ->) decode, ragged prompts and then single tokens, as a layer
    of a model runs them; the steps also replayed from one captured graph, on a stream of its own."""
    g = gen(81)
    page, Hq, H, d, steps = 16, 8, 2, 128, 20
    prompts = [70, 1, 133]
    final = [n + steps for n in prompts]
    pool, table, _ = make(BF16, kind, final, page, Hq, H, d, g)
    t = table.to(DEV)
    freq = (1e4 ** (-torch.arange(0, d, 2).double() / d)).float()
    qw, kw = [(1 + torch.randn(d, generator=g) / 8).to(BF16) for _ in range(2)]
    wide = [torch.randn(n, Hq + 2 * H, d, generator=g).to(BF16) for n in final]
    fd, qwd, kwd = freq.to(DEV), qw.to(DEV), kw.to(DEV)
    x = torch.cat([w[:n] for w, n in zip(wide, prompts)]).to(DEV)
    pos = torch.cat([torch.arange(n) for n in prompts]).to(torch.int32).to(DEV)
    _, k = norm_rope(x[:, :Hq], x[:, Hq:Hq + H], pos, fd, qwd, kwd)
    pool.append(0, k, x[:, Hq + H:].contiguous(), dev_lens(prompts), t, cu_of(prompts).to(DEV), max(prompts))
    lens = dev_lens(prompts)
    x = torch.empty(3, Hq + 2 * H, d, dtype=BF16, device=DEV)
    out, sparse = [torch.empty(3, Hq, d, dtype=BF16, device=DEV) for _ in range(2)]
    sel = torch.empty(3, H, 6, dtype=torch.int32, device=DEV)
    v = torch.empty(3, H, d, dtype=BF16, device=DEV)
    q_rot = torch.empty(3, Hq, d, dtype=BF16, device=DEV)

    def step():
        lens.add_(1)
        q, k = norm_rope(x[:, :Hq], x[:, Hq:Hq + H], lens - 1, fd, qwd, kwd, q_out=q_rot)
        v.copy_(x[:, Hq + H:])
        pool.append(0, k, v, lens, t)
        pool.decode(0, q, lens, t, max(final), out)
        pool.select(0, q, lens, t, max(final), 1, 2, 3, sel)
        pool.decode(0, q, lens, t, max(final), sparse, selected=sel)

    graph = None
    ks = [ref.norm_rope(w[:, Hq:Hq + H], kw, torch.arange(w.shape[0]), freq, 1e-6, False)[0] for w in wide]
    for i in range(steps):
        x.copy_(torch.stack([w[n + i] for w, n in zip(wide, prompts)]))
        if captured and i == 3:
            torch.cuda.synchronize()
            graph, keep = torch.cuda.CUDAGraph(), lens.clone()
            with torch.cuda.graph(graph):
                step()
            assert torch.equal(lens, keep)
        if graph is not None:
            graph.replay()
        else:
            step()
        if i in (0, 2, 3, 9, steps - 1):
            torch.cuda.synchronize()
            for b, n in enumerate(prompts):
                m = n + i + 1
                # the rows as the pool holds them: their own accuracy is tested above
                ko, vo = torch.empty(m, H, d, dtype=BF16, device=DEV), torch.empty(m, H, d, dtype=BF16, device=DEV)
                one = lambda z: z[b:b + 1].contiguous()
                pool.read(0, one(lens), one(t), ko, vo, cu_of([m]).to(DEV))
                kk, vv = ko.double().cpu(), vo.double().cpu()
                if kind == BF16:
                    assert float((kk - ks[b][:m]).abs().max()) < 0.05
                else:                                          # rounding to 16 bits on the way out is not in the attention
                    pages, slot = table[b, torch.arange(m) // page].long(), torch.arange(m) % page
                    rows = lambda z, s: z[0].view(torch.int8).cpu()[pages, :, slot].view(E4M3).double() * s[0].cpu()[pages, :, slot].double()[..., None]
                    kk, vv = rows(pool.k, pool.k_scale), rows(pool.v, pool.v_scale)
                o, _, ob, _ = ref.attention(q_rot[b].cpu(), kk.transpose(0, 1), vv.transpose(0, 1), BF16, kind=kind)
                within(out[b], o, ob, (i, b))
                want = sel[b].tolist()
                for h in range(H):
                    at = [r for p in want[h] if p >= 0 for r in range(p * page, min(m, (p + 1) * page))]
                    G = Hq // H
                    o, _, ob, _ = ref.attention(q_rot[b, h * G:(h + 1) * G].cpu(), kk.transpose(0, 1)[h:h + 1, at], vv.transpose(0, 1)[h:h + 1, at], BF16, kind=kind)
                    within(sparse[b, h * G:(h + 1) * G], o, ob, (i, b, h))
    assert pool.status() == 0


def test_two_streams_at_once(cuda_device):
    """Two decodes of one pool in flight on two streams: neither sees the other's workspace."""
    pool, table, ks, vs, q, out = attend_case(BF16, BF16, [20000], 16, 8, 1, 128, 91)
    qd, lens, t = q.to(DEV), dev_lens([20000]), table.to(DEV)
    q2 = torch.randn_like(qd)
    want = torch.empty_like(out)
    pool.decode(1, q2, lens, t, 20000, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty(20, *out.shape, dtype=BF16, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(20):
        for s, x, o in zip(streams, (qd, q2), outs):
            pool.decode(1, x, lens, t, 20000, o[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[0][i], out) and torch.equal(outs[1][i], want) for i in range(20))


def test_streams_ordered_by_events(cuda_device):
    """Rows appended on one stream and attended to on another, ordered by events alone, every step a little longer; the
    steps' results are those of one stream."""
    g = gen(93)
    steps, H, d = 40, 4, 64
    pool, table, _ = make(BF16, E4M3, [steps], 16, 8, H, d, g)
    t = table.to(DEV)
    k, v = [torch.randn(steps, H, d, generator=g).to(BF16).to(DEV) for _ in range(2)]
    q = torch.randn(steps, 1, 8, d, generator=g).to(BF16).to(DEV)
    lens = [dev_lens([i + 1]) for i in range(steps)]
    want, got = torch.empty_like(q), torch.empty_like(q)
    for i in range(steps):
        pool.append(0, k[i:i + 1], v[i:i + 1], lens[i], t)
        pool.decode(0, q[i], lens[i], t, steps, want[i])
    torch.cuda.synchronize()
    poison(pool)
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(steps):
        pool.append(0, k[i:i + 1], v[i:i + 1], lens[i], t, stream=a)
        b.wait_event(a.record_event())
        pool.decode(0, q[i], lens[i], t, steps, got[i], stream=b)
        a.wait_event(b.record_event())
    torch.cuda.synchronize()
    assert pool.status() == 0 and torch.equal(got, want)


def test_paged_and_bounded_steps_in_turn(cuda_device):
    """Decode steps of bounded caches (which start early behind one another) between steps of a paged one: both as alone."""
    from tests.harness import make_buzz
    import workloads
    w = workloads.scaled(workloads.get("C4"), layers=3, batch=2, q_heads=8, kv_heads=2, prompt_min=300, prompt_max=300, decode_steps=30, window=64, budget=512)
    outs = []
    for mixed in (False, True):
        bz = make_buzz(w)
        g = gen(94)
        pool, table, _ = make(BF16, BF16, [40, 40], 32, 8, 2, 128, g)
        t = table.to(DEV)
        steps = [workloads.decode_inputs(w, l, DEV) for l in range(3)]
        for l in range(3):
            q, k, v, cu = workloads.prefill_inputs(w, l, DEV)
            bz.prefill(l, q, k, v, cu, 300, torch.empty_like(q))
        a, p = torch.empty(30, 3, 2, 8, 128, dtype=BF16, device=DEV), torch.empty(30, 3, 2, 8, 128, dtype=BF16, device=DEV)
        lens = [dev_lens([i + 1] * 2) for i in range(30)]

        def paged(i, l):
            pool.append(l % 2, steps[l][1][i], steps[l][2][i], lens[i], t)
            pool.decode(l % 2, steps[l][0][i], lens[i], t, 40, p[i, l])

        torch.cuda.synchronize()
        for i in range(30):
            for l in range(3):
                bz.decode_step(l, steps[l][0][i], steps[l][1][i], steps[l][2][i], a[i, l])
                if mixed:
                    paged(i, l)
        if not mixed:
            for i in range(30):
                for l in range(3):
                    paged(i, l)
        assert bz.status() == 0 and pool.status() == 0
        outs.append((a, p))
        bz.close()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_paged_and_bounded_caches_side_by_side(cuda_device):
    """While nothing has been evicted, a bounded cache and a paged one of the same layer give the same attention."""
    from tests.harness import make_buzz
    import workloads
    w = workloads.scaled(workloads.get("C4"), layers=1, batch=2, q_heads=8, kv_heads=2, prompt_min=200, prompt_max=200, decode_steps=4, window=64, budget=512)
    bz = make_buzz(w)
    q, k, v, cu = workloads.prefill_inputs(w, 0, DEV)
    bz.prefill(0, q, k, v, cu, 200, torch.empty_like(q))
    pool, table, _ = make(BF16, BF16, [204, 204], 32, 8, 2, 128, gen(3))
    t = table.to(DEV)
    pool.append(0, k, v, dev_lens([200, 200]), t, cu, 200)
    dq, dk, dv = workloads.decode_inputs(w, 0, DEV)
    for i in range(4):
        a, b = torch.empty_like(dq[i]), torch.empty_like(dq[i])
        bz.decode_step(0, dq[i], dk[i], dv[i], a)
        lens = dev_lens([201 + i] * 2)
        pool.append(0, dk[i], dv[i], lens, t)
        pool.decode(0, dq[i], lens, t, 204, b)
        torch.testing.assert_close(a.float(), b.float(), atol=2e-2, rtol=1e-2)
    assert bz.status() == 0 and pool.status() == 0
    bz.close()
