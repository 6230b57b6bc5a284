"""The cache in pages on the GPU against its float64 oracle: writing and reading back exactly, attention within bounds
that count the roundings.

Attention's bound, element by element, with u the type's half step (fp16 2^-11, bf16 2^-8; torch.finfo(t).eps / 2):
a score is off by at most delta = reach * (D + 8) * 2^-24 (reach: the sum of |q||k| times the scale; D sums in fp32, and a few
roundings of the scale, the maximum's subtraction and the exponential's argument), which moves every weight by a factor of
at most 1 + 2 delta; a weight is rounded to the type before it multiplies a value (u) and the exponential and the division
are off by a few 2^-23; n products are summed in fp32 (n * 2^-24).  All of these count on spread = sum of weight * |v|.  The output
is rounded once more (u * |out|, or half a step of the type's smallest numbers).  A weight too small for u is rounded by half
a step of the type's subnormal numbers: fp16 weights are held times at least 2^6, the largest being 2^6 or more, so that this is
at most 2^-25 / 2^6 = 2^-31 of the largest weight and of their sum, and counts on mass = sum of |v| (bf16: 2^-134, nothing).
"""
import numpy as np
import pytest
import torch

import paper_2501_16383_amd as R
from oracle import paged_oracle as O
from paper_2501_16383_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda:0"
FORMATS = [(b, t, d) for b in (16, 8, 4) for t in ("fp16", "bf16") for d in (64, 128)]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Setup:
    """A pool whose memory holds NaN (as every format reads 0xff) outside the tokens written, sequences of the given
    lengths in pages dealt in random order, and their keys and values (host, of the type)."""

    def __init__(self, lens, hq=4, hkv=2, D=128, bits=8, dtype="fp16", page=16, seed=0, spare=3, scale_k=1.0):
        self.lens, self.hq, self.hkv, self.D, self.bits, self.dtype, self.page = list(lens), hq, hkv, D, bits, dtype, page
        self.g = torch.Generator().manual_seed(seed)
        need = [(n + page - 1) // page for n in lens]
        self.n_pages = sum(need) + spare
        self.cols = max(max(need), 1) + 1
        perm = torch.randperm(self.n_pages, generator=self.g).tolist()
        self.table = torch.full((len(lens), self.cols), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = torch.tensor(perm[at:at + n], dtype=torch.int32)
            at += n
        self.cfg = R.RkvPagedConfig(hq, hkv, self.n_pages, head_dim=D, page_tokens=page, bits=bits, dtype=0 if dtype == "fp16" else 1)
        mem = torch.full((R.paged_sizes(self.cfg),), 255, dtype=torch.uint8, device=DEV)
        self.cache = R.RkvPagedCache(self.cfg, device=DEV, mem=mem)
        self.k = [self.noise(n, hkv) * scale_k for n in lens]
        self.v = [self.noise(n, hkv) for n in lens]
        self.dtable = self.table.to(DEV)

    def noise(self, n, heads):
        x = torch.randn(n, heads, self.D, generator=self.g)
        x[..., 3] *= 8                                         # a strong channel
        return x.to(TYPES[self.dtype])

    def batch(self, lens, news, extra=0, **kw):
        """Rows of the sequences' last `news` tokens of `lens`."""
        starts = [0]
        for m in news:
            starts.append(starts[-1] + m)
        kw.setdefault("max_new", max(max(news), 1))
        return R.RkvPagedBatch(self.dtable, ints(starts), ints(lens), n_rows=starts[-1] + extra, **kw)

    def rows(self, xs, lens, news, extra=0):
        """Packed device rows of per-sequence tensors xs."""
        t = [x[max(n - m, 0):n] for x, n, m in zip(xs, lens, news)]
        t = [torch.cat([torch.full((m - len(x), *x.shape[1:]), 9.0, dtype=x.dtype), x]) for x, m in zip(t, news)]   # rows in front
        t.append(torch.full((extra, *xs[0].shape[1:]), 9.0, dtype=xs[0].dtype))
        return torch.cat(t).to(DEV)

    def fill(self, lens=None):
        lens = self.lens if lens is None else lens
        if sum(lens):
            self.cache.append(self.rows(self.k, lens, lens), self.rows(self.v, lens, lens), self.batch(lens, lens))

    def held(self, xs, b, n):
        return O.stored(xs[b][:n].double().numpy(), self.bits, self.dtype)


def check_attention(s, lens, news, got, lse=None, q=None, rows_from=0, **kw):
    u = torch.finfo(TYPES[s.dtype]).eps / 2
    tiny = 2.0 ** (-25 if s.dtype == "fp16" else -134)
    least = 2.0**-31 if s.dtype == "fp16" else 0
    row = rows_from
    got, q = got.cpu().double().numpy(), q.cpu().double().numpy()
    for b, (n, m) in enumerate(zip(lens, news)):
        ref, rl, spread, reach, mass = O.attention(q[row:row + m], s.held(s.k, b, n), s.held(s.v, b, n), n - m, **kw)
        delta = (reach * (s.D + 8) * 2.0**-24)[..., None]
        tol = spread * (u + 2 * delta + (n + 16) * 2.0**-24) * 1.001 + u * np.abs(ref) + tiny + mass * least
        err = np.abs(got[row:row + m] - ref)
        assert np.isfinite(got[row:row + m]).all(), b
        assert (err <= tol).all(), (b, n, m, (err / np.maximum(tol, 1e-300)).max())
        if lse is not None:
            l = lse[row:row + m].cpu().double().numpy()
            assert np.array_equal(l == -np.inf, rl == -np.inf)
            fin = rl != -np.inf
            assert (np.abs(l[fin] - rl[fin]) <= (delta[..., 0] + (n + 32) * 2.0**-24 + np.abs(rl) * 2.0**-22)[fin]).all()
        row += m


def run(s, lens, news, want_lse=True, fill=True, **kw):
    if fill:
        s.fill()
    q = torch.cat([s.noise(m, s.hq) for m in news]).to(DEV)
    out, lse = s.cache.attention(q, s.batch(lens, news), want_lse=True, **kw)
    check_attention(s, lens, news, out, lse if want_lse else None, q, **kw)
    return out, lse, q


# ---- writing and reading back -----------------------------------------------------------------------------

@pytest.mark.parametrize("bits,dtype,D", FORMATS)
def test_read_gives_what_the_oracle_stores(bits, dtype, D):
    """Appended in two parts, ragged, an empty sequence among them; bit for bit, and nothing else of the pool changes."""
    lens = [1, 33, 0, 70, 257]
    s = Setup(lens, hkv=3, hq=3, D=D, bits=bits, dtype=dtype, page=32)
    s.fill([0, 16, 0, 70, 200])
    news = [1, 17, 0, 0, 57]
    s.cache.append(s.rows(s.k, lens, news), s.rows(s.v, lens, news), s.batch(lens, news))
    k, v = s.cache.read(s.batch(lens, lens))
    at = 0
    for b, n in enumerate(lens):
        for x, xs in ((k, s.k), (v, s.v)):
            assert np.array_equal(x[at:at + n].cpu().double().numpy(), s.held(xs, b, n)), (b, n)
        at += n
    free = sorted(set(range(s.n_pages)) - set(s.table[s.table >= 0].tolist()))
    pages = s.cache.mem.view(s.n_pages, -1)
    assert free and (pages[free] == 255).all()


@pytest.mark.parametrize("bits,dtype", [(b, t) for b in (8, 4) for t in ("fp16", "bf16")])
def test_every_number_of_the_type(bits, dtype):
    """All 65536 bit patterns as a block's largest number, smaller ones beside them: subnormals, the largest numbers, both zeros,
    infinities and NaN."""
    t = TYPES[dtype]
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(t)
    x = x[:, None] * torch.linspace(1, 0.003, 32).to(t)[None]
    x = x.view(1024, 16, 128)
    s = Setup([1024], hq=16, hkv=16, bits=bits, dtype=dtype, page=64)
    s.k, s.v = [x], [x.flip(-1)]
    s.fill()
    k, v = s.cache.read(s.batch([1024], [1024]))
    for got, xs in ((k, s.k), (v, s.v)):
        want = s.held(xs, 0, 1024)
        assert np.array_equal(got.cpu().double().numpy(), want, equal_nan=True)
        assert np.isnan(want).any()


def test_the_pool_is_laid_out_as_documented():
    s = Setup([40], hq=2, hkv=2, D=64, bits=4, page=16)
    s.fill()
    blk = s.cache.mem.cpu().numpy().reshape(s.n_pages, 2, -1)
    for x, codes_at, scales_at in ((s.k[0], 0, 1024), (s.v[0], 512, 1056)):
        for t in (0, 15, 16, 39):
            b = blk[s.table[0, t // 16].item(), 1]
            codes = b[codes_at + (t % 16) * 32:][:32]
            nib = np.stack([codes & 15, codes >> 4], -1).reshape(-1)
            val = np.where(nib & 8, -1, 1) * O.E2M1[nib & 7]
            two = 2.0 ** (b[scales_at + (t % 16) * 2:][:2].astype(int) - 127)
            want = O.stored(x[t, 1].double().numpy()[None], 4, "fp16")[0]
            assert np.array_equal(val * np.repeat(two, 32), want)


def test_strided_rows_and_rows_of_nobody():
    """Keys and values as columns of one tensor; rows behind the last sequence stay as they were, in the pool and in what is
    read; a row in front of its sequence's first token reads as zero."""
    lens, news = [5, 20], [8, 20]
    s = Setup(lens, hq=4, hkv=2)
    qkv = torch.full((31, 8, 128), 7.0, dtype=torch.float16, device=DEV)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    k.copy_(s.rows(s.k, lens, news, extra=3))
    v.copy_(s.rows(s.v, lens, news, extra=3))
    b = s.batch(lens, news, extra=3)
    s.cache.append(k, v, b)
    back = torch.full((31, 4, 128), -3.0, dtype=torch.float16, device=DEV)
    s.cache.read(b, back[:, :2], back[:, 2:])
    assert (back[:3] == 0).all() and (back[28:] == -3).all()
    assert np.array_equal(back[3:8, :2].cpu().double().numpy(), s.held(s.k, 0, 5))
    assert np.array_equal(back[8:28, 2:].cpu().double().numpy(), s.held(s.v, 1, 20))
    out = torch.full((31, 4, 128), -3.0, dtype=torch.float16, device=DEV)
    lse = torch.full((31, 4), -3.0, device=DEV)
    qd = torch.cat([s.noise(31, 4)]).to(DEV)
    q.copy_(qd)
    s.cache.attention(q, b, out=out, lse=lse)
    assert (out[28:] == -3).all() and (lse[28:] == -3).all() and (out[:3] == 0).all() and (lse[:3] == -np.inf).all()
    check_attention(s, lens, news, out, lse, qd)


def test_pages_far_into_a_large_pool():
    """Blocks that lie past 4 GiB."""
    cfg = R.RkvPagedConfig(8, 8, 5000, page_tokens=256, bits=16, dtype=0)
    assert R.paged_sizes(cfg) > 4 << 30
    mem = torch.empty(R.paged_sizes(cfg), dtype=torch.uint8, device=DEV)
    cache = R.RkvPagedCache(cfg, device=DEV, mem=mem)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(300, 8, 128, generator=g).half().to(DEV) for _ in range(2))
    b = R.RkvPagedBatch(ints([[4999, 4097]]), ints([0, 300]), ints([300]), n_rows=300)
    cache.append(k, v, b)
    rk, rv = cache.read(b)
    assert torch.equal(rk, k) and torch.equal(rv, v)
    q = torch.randn(300, 8, 128, generator=g).half().to(DEV)
    out = cache.attention(q, b)
    small = R.RkvPagedCache(R.RkvPagedConfig(8, 8, 2, page_tokens=256, bits=16, dtype=0), device=DEV)
    b2 = R.RkvPagedBatch(ints([[1, 0]]), ints([0, 300]), ints([300]), n_rows=300)
    small.append(k, v, b2)
    assert torch.equal(out, small.attention(q, b2))


# ---- attention --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits,dtype,D", FORMATS)
def test_attention_of_a_ragged_batch(bits, dtype, D):
    """Single tokens, drafted ones, chunks and whole prompts together; an empty sequence, and one without new rows."""
    lens = [1, 17, 0, 64, 65, 130, 300, 200, 40]
    news = [1, 1, 0, 64, 3, 130, 70, 1, 0]
    run(Setup(lens, hq=8, hkv=2, D=D, bits=bits, dtype=dtype, page=16, seed=D + bits), lens, news)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (3, 1), (14, 2), (16, 1), (17, 1), (40, 1), (80, 2)])
@pytest.mark.parametrize("bits,D", [(8, 128), (16, 64)])
def test_attention_of_head_layouts(hq, hkv, bits, D):
    lens, news = [90, 33, 5], [1, 4, 5]
    run(Setup(lens, hq=hq, hkv=hkv, D=D, bits=bits, dtype="bf16", page=32, seed=hq), lens, news)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("news", [[1, 1, 1], [2, 150, 31]], ids=str)
def test_attention_of_page_sizes(page, news):
    lens = [259, 511, 31]
    run(Setup(lens, hq=4, hkv=1, page=page, bits=4 if page == 64 else 8, seed=page), lens, news)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 7, 64, 100, 4000])
@pytest.mark.parametrize("news", [[1, 1, 1], [40, 170, 300]], ids=str)
def test_windows_and_direction(causal, window, news):
    lens = [40, 333, 300]
    run(Setup(lens, hq=4, hkv=2, bits=8, seed=window), lens, news, causal=causal, window=window)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 255, 257])
def test_lengths_around_the_tiles(n):
    """As many rows as tokens, and one row of as many tokens."""
    s = Setup([n, n], hq=2, hkv=1, bits=16, page=16, seed=n)
    run(s, [n, n], [n, 1])


@pytest.mark.parametrize("bits,dtype,D,new", [(8, "bf16", 128, 1), (4, "fp16", 64, 1), (16, "fp16", 128, 3), (8, "fp16", 128, 40), (8, "bf16", 64, 130)])
def test_long_sequences(bits, dtype, D, new):
    lens, news = [20011, 777], [new, 1]
    run(Setup(lens, hq=2, hkv=1, D=D, bits=bits, dtype=dtype, page=64, seed=new), lens, news)


@pytest.mark.parametrize("bits,D", [(16, 128), (8, 64), (4, 128)])
@pytest.mark.parametrize("news", [[4, 1, 2, 4], [5, 8, 1, 7], [9, 5, 4, 1], [64, 8, 4, 1], [65, 7, 1, 128]], ids=str)
def test_columns_around_the_kernels_bounds(bits, D, news):
    """16, 32, 36, 256 and 260 columns of a KV head and few beside them, over enough tokens to be cut into splits."""
    run(Setup([1400, 900, 700, 333], hq=4, hkv=1, D=D, bits=bits, dtype="bf16", page=16, seed=sum(news)), [1400, 900, 700, 333], news)


@pytest.mark.parametrize("window", [0, 50, 700])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new", [1, 3, 90, 300])
def test_tables_far_wider_than_the_sequences(window, causal, new):
    """Without max_len the host cuts the table's capacity into splits: of these sequences most are empty."""
    s = Setup([600, 310], hq=2, hkv=1, seed=new)
    s.dtable = torch.cat([s.dtable, torch.full((2, 4000), 2**30, dtype=torch.int32, device=DEV)], 1)
    run(s, [600, 310], [new, 1], causal=causal, window=window)


@pytest.mark.parametrize("causal", [True, False])
def test_more_rows_than_tokens(causal):
    """Rows in front of the first token see nothing, whatever the direction."""
    out, lse, _ = run(Setup([40, 3, 0], hq=4, hkv=2, seed=3), [40, 3, 0], [100, 5, 7], causal=causal)
    assert (out[:60] == 0).all() and (lse[:60] == -np.inf).all() and (out[60:100] != 0).any() and (lse[105:] == -np.inf).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_a_page_outside_the_pool_in_a_long_sequence(bits):
    """Splits whose pages are in order, and one whose are not, meet."""
    lens, news = [3000, 2000], [40, 1]
    s = Setup(lens, hq=4, hkv=2, bits=bits, page=32, seed=6)
    out0, _, q = run(s, lens, news)
    s.dtable[1, 20] = s.n_pages
    out = s.cache.attention(q, s.batch(lens, news))
    assert torch.equal(out[:40], out0[:40]) and torch.isnan(out[40]).all()
    s.dtable[0, 92] = -1                                       # tokens 2944 .. 2975: rows 0 ..: every row but those before 2944
    assert torch.isnan(s.cache.attention(q, s.batch(lens, news))).all()
    s.dtable[0, 92], s.dtable[0, 93] = s.table[0, 92], -1      # tokens 2976 ..: from row 16 on
    out = s.cache.attention(q, s.batch(lens, news))
    assert torch.equal(out[:16], out0[:16]) and torch.isnan(out[16:40]).all()


def test_output_in_the_queries_place():
    lens, news = [700, 300], [90, 2]
    s = Setup(lens, hq=4, hkv=2, seed=5)
    out0, _, q = run(s, lens, news)
    assert s.cache.attention(q, s.batch(lens, news), out=q) is q and torch.equal(q, out0)


def test_many_sequences():
    lens = [(7 * i) % 50 for i in range(300)]
    news = [min(n, 1 + (i % 3 == 0) * (i % 20)) for i, n in enumerate(lens)]
    run(Setup(lens, hq=2, hkv=1, D=64, seed=5), lens, news)


def test_strong_scores_and_other_scales():
    """A softmax that is nearly all on one token, one that is flat, and a negative scale."""
    lens, news = [300, 90], [60, 1]
    for scale in (1.0, 0.0, -0.3, 1e-4):
        run(Setup(lens, bits=16, scale_k=2.0, seed=1), lens, news, scale=scale)


@pytest.mark.parametrize("bits,dtype", [(16, "fp16"), (16, "bf16"), (8, "fp16"), (4, "bf16")])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_a_row_does_not_see_has_no_influence(bits, dtype, bad):
    """Infinities and NaN in keys and values of later tokens: the rows in front give the bits they give without them, and
    rows that see a NaN are NaN."""
    lens, news = [150, 40], [100, 1]
    clean = Setup(lens, hq=4, hkv=2, bits=bits, dtype=dtype, seed=9)
    out0, lse0, q = run(clean, lens, news)
    s = Setup(lens, hq=4, hkv=2, bits=bits, dtype=dtype, seed=9)
    s.k[0][120, 0, 5] = bad                                    # positions 120 and 130 of the first sequence: rows 70, 80
    s.v[0][130, 1, 64] = bad
    s.fill()
    out, lse = s.cache.attention(q, s.batch(lens, news), want_lse=True)
    assert torch.equal(out[:70], out0[:70]) and torch.equal(lse[:70], lse0[:70])
    assert torch.equal(out[100], out0[100])
    first = out[:, :2]                                         # query heads of KV head 0: its values are clean
    assert torch.equal(out[70:80, 2:], out0[70:80, 2:]) and torch.equal(lse[:, 2:], lse0[:, 2:])
    channel = slice(64, 65) if bits == 16 else slice(64, 96)   # quantised: the whole block
    assert not torch.isfinite(out[80:100, 2:, channel]).any()
    rest = torch.ones(128, dtype=torch.bool)
    rest[channel] = False
    assert torch.equal(out[80:100, 2:][..., rest], out0[80:100, 2:][..., rest])
    if bits < 16 or np.isnan(bad):
        assert torch.isnan(first[70:100]).all() and torch.isnan(lse[70:100, :2]).all()


def test_scores_of_minus_infinity():
    """Keys of -infinity: a row that sees only those gets zeros, others are as without them."""
    s = Setup([30], hq=1, hkv=1, bits=16, seed=2)
    s.k[0][:10] = 0
    s.k[0][:10, 0, 0] = -np.inf
    s.fill()
    q = s.noise(30, 1)
    q[:, 0, 0] = 1.0
    out, lse = s.cache.attention(q.to(DEV), s.batch([30], [30]), want_lse=True)
    assert (out[:10] == 0).all() and (lse[:10] == -np.inf).all()
    assert torch.isfinite(out[10:]).all() and torch.isfinite(lse[10:]).all()
    s.k[0], s.v[0] = s.k[0][10:], s.v[0][10:]
    check_attention(s, [20], [20], out[10:], lse[10:], q[10:])


def test_queries_that_are_not_finite_touch_only_their_row():
    lens, news = [100, 100], [50, 1]
    s = Setup(lens, hq=4, hkv=1, seed=4)
    out0, _, q = run(s, lens, news)
    q[20, 2, 7], q[50, 1, 0] = np.nan, np.nan
    out = s.cache.attention(q, s.batch(lens, news))
    same = torch.ones(51, 4, dtype=torch.bool)
    same[20, 2] = same[50, 1] = False
    assert torch.equal(out[same], out0[same]) and torch.isnan(out[~same]).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_a_scale_of_zero(dtype):
    """Every score that is a number counts as 0, one of a query that is not finite is NaN, whichever kernel a sequence goes to;
    bf16 queries whose products with the keys would pass fp32 are numbers."""
    lens, news = [300, 90], [60, 2]                            # 240 columns, and 8
    far = dtype == "bf16"
    s = Setup(lens, hq=4, hkv=1, bits=16, dtype=dtype, scale_k=2.0**60 if far else 1.0, seed=1)
    s.fill()
    q = torch.cat([s.noise(m, 4) for m in news])
    if far:
        q[[25, 60]] = 2.0**100
    clean = q.clone()
    for row in (20, 61):
        q[row, 0, 7], q[row, 1, 0], q[row, 2, 63] = np.nan, np.inf, -np.inf
    out, lse = s.cache.attention(q.to(DEV), s.batch(lens, news), scale=0.0, want_lse=True)
    odd = torch.zeros(62, 4, dtype=torch.bool)
    odd[20, :3] = odd[61, :3] = True
    assert torch.isnan(out[odd]).all() and torch.isnan(lse[odd]).all()
    want, wl = s.cache.attention(torch.zeros_like(clean).to(DEV), s.batch(lens, news), scale=1.0, want_lse=True)
    check_attention(s, lens, news, want, wl, torch.zeros_like(clean))
    assert torch.equal(out[~odd], want[~odd]) and torch.equal(lse[~odd], wl[~odd])


@pytest.mark.parametrize("news", [[3, 1], [10, 1], [20, 1], [70, 2]], ids=str)
@pytest.mark.parametrize("bits,dtype,D,e,scale", [(16, t, 64, e, np.log(2)) for t in ("fp16", "bf16") for e in (20, 23, 24, 25, 26, 27, 28)]
                         + [(b, t, 64 if b == 8 else 128, e, np.log(2)) for b in (8, 4) for t in ("fp16", "bf16") for e in (24, 27)]
                         + [(16, "fp16", 128, 29, 1.0), (16, "fp16", 64, 29, -1.0), (8, "bf16", 128, 33, 1.0), (16, "bf16", 128, 40, 1.0)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_so_large_that_fp32_holds_few_of_them(bits, dtype, D, e, scale, news, sign):
    """Scores 2^e + j 2^(e - 23), or less than 0 by as much: neighbours in fp32, from two channels whose products and sum are exact.  With a scale of log(2), a
    power of two's exponent is the score itself, so that the weights are exact powers; with 1, whose scaled scores are rounded, j goes in steps of 4:
    two scores are the same or further apart than any weight reaches.  So no error of a score counts in the bound, and what a
    weight's rounding to fp16's subnormal numbers costs is at most 2^-25 of the largest weight, which is 1 or more (header).
    Rows of small queries stand among them and have the bits that they have alone."""
    lens, kw = [700, 130], dict(scale=scale, window=90 if e % 2 else 0)
    s = Setup(lens, hq=2, hkv=1, D=D, bits=bits, dtype=dtype, seed=e)
    for k in s.k:
        k.zero_()
        k[:, 0, 0] = 2.0 ** (e - e // 2)
        k[:, 0, 40] = torch.randint(0, 8, k.shape[:1], generator=s.g).to(k.dtype) * (1 if abs(scale) < 1 else 4)
    s.fill()
    q = torch.zeros(sum(news), 2, D, dtype=TYPES[dtype])
    q[..., 0], q[..., 40] = 2.0 ** (e // 2) * np.sign(scale) * sign, 2.0 ** (e - 23) * np.sign(scale) * sign
    near = q * 2.0**-30
    out, lse = (x.cpu().double().numpy() for x in s.cache.attention(q.to(DEV), s.batch(lens, news), want_lse=True, **kw))
    u, least = (2.0**-11, 2.0**-25) if dtype == "fp16" else (2.0**-8, 0)
    row = 0
    for b, (n, m) in enumerate(zip(lens, news)):
        ref, rl, spread, _, mass = O.attention(q[row:row + m].double().numpy(), s.held(s.k, b, n), s.held(s.v, b, n), n - m, **kw)
        assert np.isfinite(out[row:row + m]).all() and np.isfinite(lse[row:row + m]).all()
        tol = spread * (u + (n + 16) * 2.0**-24) * 1.001 + u * np.abs(ref) + 2.0**-25 + mass * least
        assert (np.abs(out[row:row + m] - ref) <= tol).all(), (b, (np.abs(out[row:row + m] - ref) / tol).max())
        assert (np.abs(lse[row:row + m] - rl) <= np.abs(rl) * 2.0**-22).all()
        row += m
    few = torch.arange(sum(news)) % 3 != 1
    mixed = torch.where(few[:, None, None], q, near).to(DEV)
    a, b = (s.cache.attention(x, s.batch(lens, news), want_lse=True, **kw) for x in (mixed, near.to(DEV)))
    assert torch.equal(a[0][~few], b[0][~few]) and torch.equal(a[1][~few], b[1][~few])
    assert np.array_equal(a[0][few].cpu().double().numpy(), out[few.numpy()])


@pytest.mark.parametrize("news", [[1, 1], [12, 1], [40, 1]], ids=str)
@pytest.mark.parametrize("step", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype,e", [("fp16", 22), ("fp16", 24), ("fp16", 25), ("fp16", 26), ("fp16", 27), ("fp16", 28), ("bf16", 27)])
def test_large_scores_that_grow(dtype, e, step, news):
    """As above, the scores growing by `step` of fp32's neighbours every 128 tokens, so that every tile of a wave has a new maximum just above the
    one before; up to 512 tokens, which one workgroup walks."""
    lens = [500, 512]
    s = Setup(lens, hq=2, hkv=1, D=64, bits=16, dtype=dtype, seed=e)
    for k in s.k:
        k.zero_()
        k[:, 0, 0] = 2.0 ** (e - e // 2)
        k[:, 0, 40] = torch.arange(k.shape[0]).div(128, rounding_mode="floor").to(k.dtype) * step
    s.fill()
    q = torch.zeros(sum(news), 2, 64, dtype=TYPES[dtype])
    q[..., 0], q[..., 40] = 2.0 ** (e // 2), 2.0 ** (e - 23)
    out, lse = (x.cpu().double().numpy() for x in s.cache.attention(q.to(DEV), s.batch(lens, news, max_len=512), scale=np.log(2), want_lse=True))
    u, least = (2.0**-11, 2.0**-25) if dtype == "fp16" else (2.0**-8, 0)
    row = 0
    for b, (n, m) in enumerate(zip(lens, news)):
        ref, rl, spread, _, mass = O.attention(q[row:row + m].double().numpy(), s.held(s.k, b, n), s.held(s.v, b, n), n - m, scale=np.log(2))
        tol = spread * (u + (n + 16) * 2.0**-24) * 1.001 + u * np.abs(ref) + 2.0**-25 + mass * least
        assert np.isfinite(out[row:row + m]).all() and (np.abs(out[row:row + m] - ref) <= tol).all(), b
        assert (np.abs(lse[row:row + m] - rl) <= np.abs(rl) * 2.0**-22).all()
        row += m


def test_large_scores_and_what_is_no_number():
    """Rows whose scores are large, over a page outside the pool, a NaN key and an infinite one: NaN from there on, and the rows in front
    and the other KV head's as they are without."""
    lens, news = [300, 40], [90, 1]
    made = [Setup(lens, hq=4, hkv=2, bits=16, seed=2, scale_k=64.0) for _ in range(2)]
    for s in made:
        s.fill()
    s = made[0]
    q = (torch.cat([s.noise(m, 4) for m in news]) * 2048.0).to(DEV)
    out0, lse0 = s.cache.attention(q, s.batch(lens, news), scale=16.0, want_lse=True)
    assert torch.isfinite(out0).all() and torch.isfinite(lse0).all() and (lse0.abs() > 2**20).any()
    s.dtable[0, 16] = -1                                       # tokens 256 ..: rows 46 ..
    out, lse = s.cache.attention(q, s.batch(lens, news), scale=16.0, want_lse=True)
    assert torch.equal(out[:46], out0[:46]) and torch.equal(lse[:46], lse0[:46]) and torch.isnan(out[46:90]).all() and torch.isnan(lse[46:90]).all()
    assert torch.equal(out[90], out0[90])
    for bad in (np.nan, np.inf):
        s = made[1]
        s.k[0][256, 0, 5] = bad
        s.fill()
        out, lse = s.cache.attention(q.abs(), s.batch(lens, news), scale=16.0, want_lse=True)
        want, wl = made[0].cache.attention(q.abs(), R.RkvPagedBatch(made[0].table.to(DEV), ints([0, 90, 91]), ints(lens), 91, max_new=90), scale=16.0,
                                           want_lse=True)
        assert torch.equal(out[:46], want[:46]) and torch.equal(lse[:46], wl[:46]) and torch.equal(out[:, 2:], want[:, 2:])
        assert torch.isnan(out[46:90, :2]).all() and torch.isnan(lse[46:90, :2]).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("long", [False, True], ids=["whole", "splits"])
@pytest.mark.parametrize("news", [[5, 1], [14, 2], [8, 40]], ids=str)
@pytest.mark.parametrize("bits,dtype,D", [(16, "fp16", 128), (16, "bf16", 64), (8, "bf16", 128), (8, "fp16", 64), (4, "fp16", 128), (4, "bf16", 64)])
def test_what_drafted_tokens_do_not_see(bits, dtype, D, news, long, bad):
    """As above for few rows: up to 16 and 32 columns and beside a chunk, in one span and in splits.  The spoilt key and value lie between the
    first and the last new row's positions."""
    lens = [1401, 700] if long else [150, 90]
    made = [Setup(lens, hq=4, hkv=2, D=D, bits=bits, dtype=dtype, seed=9) for _ in range(2)]
    n, m = lens[0], news[0]
    made[1].k[0][n - 3, 0, 5] = bad                            # rows m - 3 .. see it
    made[1].v[0][n - 2, 1, 40] = bad                           # rows m - 2 ..
    out0, lse0, q = run(made[0], lens, news)
    s = made[1]
    s.fill()
    out, lse = s.cache.attention(q, s.batch(lens, news), want_lse=True)
    assert torch.equal(out[:m - 3], out0[:m - 3]) and torch.equal(lse[:m - 3], lse0[:m - 3])
    assert torch.equal(out[m:], out0[m:]) and torch.equal(lse[m:], lse0[m:])
    assert torch.equal(out[m - 3, 2:], out0[m - 3, 2:]) and torch.equal(lse[:, 2:], lse0[:, 2:])
    channel = slice(40, 41) if bits == 16 else slice(32, 64)
    rest = torch.ones(D, dtype=torch.bool)
    rest[channel] = False
    assert not torch.isfinite(out[m - 2:m, 2:, channel]).any()
    assert torch.equal(out[m - 2:m, 2:][..., rest], out0[m - 2:m, 2:][..., rest])
    if bits < 16 or np.isnan(bad):
        assert torch.isnan(out[m - 3:m, :2]).all() and torch.isnan(lse[m - 3:m, :2]).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bits,dtype", [(16, "fp16"), (8, "bf16"), (4, "fp16")])
@pytest.mark.parametrize("news", [[8, 1], [15, 2], [70, 5]], ids=str)
def test_what_a_window_has_left_has_no_influence(news, bits, dtype, causal):
    """A NaN key and an infinite value: rows whose window starts behind them, and, causal, rows in front of them, have the bits that they
    have without."""
    lens, window = [330, 200], 3 if news[0] < 20 else 20
    made = [Setup(lens, hq=4, hkv=2, bits=bits, dtype=dtype, seed=4) for _ in range(2)]
    n, m = lens[0], news[0]
    at = n - m + 2
    made[1].k[0][at, 0, 5], made[1].v[0][at, 1, 40] = np.nan, np.inf
    out0, lse0, q = run(made[0], lens, news, causal=causal, window=window)
    s = made[1]
    s.fill()
    out, lse = s.cache.attention(q, s.batch(lens, news), causal=causal, window=window, want_lse=True)
    first, behind = 2 if causal else 0, 2 + window             # rows first .. behind - 1 see token `at`
    clean = torch.ones(sum(news), dtype=torch.bool)
    clean[first:behind] = False
    assert clean[:m].any() and torch.equal(out[clean], out0[clean]) and torch.equal(lse[clean], lse0[clean])
    assert torch.isnan(out[first:behind, :2]).all() and not torch.isfinite(out[first:behind, 2:, 40]).any()


def test_pages_outside_the_pool():
    """Tokens of such pages are not written and read as NaN; rows that see them are NaN, the others are not touched."""
    lens, news = [100, 50], [60, 1]
    s = Setup(lens, hq=4, hkv=2, seed=6)
    out0, lse0, q = run(s, lens, news)
    for bad in (-1, s.n_pages, 2**31 - 1, -2**31):
        s.dtable = s.table.to(DEV)
        s.dtable[0, 4] = bad                                   # tokens 64 .. 79: rows 24 ..
        before = s.cache.mem.clone()
        b = s.batch(lens, news)
        s.cache.append(s.rows(s.k, lens, news), s.rows(s.v, lens, news), b)
        assert torch.equal(before, s.cache.mem)
        k, v = s.cache.read(b)
        assert torch.isnan(k[24:40]).all() and torch.isnan(v[24:40]).all() and torch.isfinite(k[:24]).all() and torch.isfinite(v[40:]).all()
        out, lse = s.cache.attention(q, b, want_lse=True)
        assert torch.equal(out[:24], out0[:24]) and torch.isnan(out[24:60]).all() and torch.equal(out[60], out0[60])
        assert torch.equal(lse[:24], lse0[:24]) and torch.isnan(lse[24:60]).all()
        one = s.cache.attention(q[-2:], s.batch(lens, [1, 1]), want_lse=True)
        assert torch.isnan(one[0][0]).all() and torch.equal(one[0][1], out0[60]) and torch.isnan(one[1][0]).all()


@pytest.mark.parametrize("what", ["length", "negative", "rows"])
def test_sequences_beyond_the_hosts_bounds(what):
    lens, news = [100, 50, 60], [5, 1, 2]
    s = Setup(lens, hq=4, hkv=2, seed=7)
    out0, lse0, q = run(s, lens, news)
    kw = dict(max_len=99) if what == "length" else dict(max_new=4) if what == "rows" else {}
    b = s.batch([-3 if what == "negative" else 100, 50, 60], news, **kw)
    before = s.cache.mem.clone()
    s.cache.append(s.rows(s.k, lens, news) * 2, s.rows(s.v, lens, [5, 0, 0], 3), R.RkvPagedBatch(s.dtable, ints([0, 5, 5, 5]), b.lengths, 8, **kw)
                   if what != "rows" else R.RkvPagedBatch(s.dtable, ints([0, 5, 5, 5]), b.lengths, 8, max_new=4))
    assert torch.equal(before, s.cache.mem)
    k, v = s.cache.read(b)
    assert torch.isnan(k[:5]).all() and torch.isnan(v[:5]).all() and torch.isfinite(k[5:]).all()
    out, lse = s.cache.attention(q, b, want_lse=True)
    assert torch.isnan(out[:5]).all() and torch.isnan(lse[:5]).all() and torch.equal(out[5:], out0[5:]) and torch.equal(lse[5:], lse0[5:])


@pytest.mark.parametrize("what", ["length", "negative", "rows"])
@pytest.mark.parametrize("news,which", [([150, 1, 5], 0), ([150, 1, 5], 2), ([90, 40, 2], 1), ([100, 4, 7], 1), ([9, 1, 4], 0), ([1, 10, 4], 1), ([3, 2, 5], 2),
                                        ([150], 0), ([6], 0)], ids=str)
def test_sequences_beyond_the_hosts_bounds_in_every_kernel(news, which, what):
    """Three columns a row, which tiles of 256 do not divide; spans that are cut into splits; the bad sequence in either kernel and alone.
    Its rows are NaN, its neighbours' as they are without it, rows of nobody untouched."""
    lens = [1400, 1333, 1290][:len(news)]
    s = Setup(lens, hq=6, hkv=2, bits=8, page=32, seed=sum(news))
    s.fill()
    told, kw = list(lens), dict(max_len=1400, max_new=max(news))
    if what == "rows":                                         # one row more than the host said; the others keep to it
        kw["max_new"] = news[which] - 1
        news = [m if b == which else min(m, kw["max_new"]) for b, m in enumerate(news)]
    else:
        told[which] = 1401 if what == "length" else -2
    q = torch.cat([s.noise(m, 6) for m in news] + [s.noise(3, 6)]).to(DEV)
    out = torch.full_like(q, 5.0)
    lse = torch.full(q.shape[:2], 5.0, device=DEV)
    s.cache.attention(q, s.batch(told, news, extra=3, **kw), out=out, lse=lse)
    row = 0
    for b, m in enumerate(news):
        if b == which:
            assert torch.isnan(out[row:row + m]).all() and torch.isnan(lse[row:row + m]).all()
        else:
            one = [m if c == b else 0 for c in range(len(news))]
            check_attention(s, lens, one, out, lse, q, rows_from=row)
        row += m
    assert (out[row:] == 5).all() and (lse[row:] == 5).all()
    if what != "rows":                                         # the same launch without the fault
        good, gl = s.cache.attention(q, s.batch(lens, news, extra=3, **kw), want_lse=True)
        keep = torch.ones(row, dtype=torch.bool)
        keep[sum(news[:which]):sum(news[:which + 1])] = False
        assert torch.equal(out[:row][keep], good[:row][keep]) and torch.equal(lse[:row][keep], gl[:row][keep])


def test_row_starts_that_make_no_sense():
    """Nothing is written out of place: what a sequence does not own stays as it was."""
    lens = [100, 50, 60]
    s = Setup(lens, seed=7)
    s.fill()
    q = s.noise(20, 4).to(DEV)
    kv = s.noise(20, 2).to(DEV)
    for starts in ([0, 30, 10, 20], [-5, 3, 8, 1000], [20, 20, 20, 20], [7, 3, 2, 1], [2**31 - 1, -2**31, 5, 9]):
        b = R.RkvPagedBatch(s.dtable, ints(starts), ints(lens), n_rows=20)
        guard = torch.full((22, 4, 128), 5.0, dtype=torch.float16, device=DEV)
        s.cache.append(kv, kv, b)
        s.cache.read(b)
        s.cache.attention(q, b, out=guard[1:21])
        assert (guard[0] == 5).all() and (guard[21] == 5).all()


def test_two_sequences_that_share_pages():
    """A common prefix is stored once."""
    s = Setup([64, 20], hq=4, hkv=2, seed=8)
    s.fill()
    table = s.table.clone()
    table[1, 2:4], table[1, :2] = table[1, :2].clone(), table[0, :2]   # 32 tokens of the first, then 20 of its own
    s.dtable = table.to(DEV)
    s.k[1], s.v[1] = (torch.cat([x[0][:32], x[1]]) for x in (s.k, s.v))
    run(s, [64, 52], [64, 20], fill=False)
    run(s, [64, 52], [1, 1], fill=False)


# ---- as a program uses them -------------------------------------------------------------------------------

@pytest.mark.parametrize("bits,dtype", [(16, "bf16"), (8, "fp16"), (4, "fp16")])
def test_prompts_in_chunks_then_tokens(bits, dtype):
    """A server's life: prompts enter in pieces while others decode; after every step the new rows are as the oracle says."""
    lens = [150, 61, 90]
    s = Setup(lens, hq=4, hkv=2, bits=bits, dtype=dtype, seed=11)
    have = [0, 0, 0]
    for news in ([64, 0, 33], [64, 60, 1], [22, 1, 50], [0, 0, 5], [0, 0, 1]):
        have = [h + n for h, n in zip(have, news)]
        b = s.batch(have, news)
        s.cache.append(s.rows(s.k, have, news), s.rows(s.v, have, news), b)
        q = torch.cat([s.noise(m, s.hq) for m in news]).to(DEV)
        out, lse = s.cache.attention(q, b, want_lse=True)
        check_attention(s, have, news, out, lse, q)
    assert have == lens


def test_the_same_call_gives_the_same_bits():
    lens, news = [3000, 900, 77], [1, 40, 77]
    s = Setup(lens, hq=8, hkv=2, seed=12)
    s.fill()
    q = torch.cat([s.noise(m, 8) for m in news]).to(DEV)
    a = s.cache.attention(q, s.batch(lens, news), want_lse=True)
    for _ in range(5):
        b = s.cache.attention(q, s.batch(lens, news), want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("news", [[1, 1], [3, 40]], ids=str)
def test_captured_steps_follow_the_lengths(news):
    """A step (append, attention) in a graph; between replays the lengths, rows and page table change in place, and the program
    does work of its own."""
    lens = [700, 90]
    s = Setup(lens, hq=8, hkv=2, bits=8, seed=13)
    s.fill([n - 8 * m if n > 8 * m else 0 for n, m in zip(lens, news)])
    have = [max(n - 8 * m, 0) for n, m in zip(lens, news)]
    table, dlen = s.dtable, ints([h + m for h, m in zip(have, news)])
    b = s.batch(lens, news, max_len=704)
    b.lengths.copy_(dlen)
    n = sum(news)
    k, v = (torch.zeros(n, 2, 128, dtype=torch.float16, device=DEV) for _ in range(2))
    q, out = torch.zeros(n, 8, 128, dtype=torch.float16, device=DEV), torch.zeros(n, 8, 128, dtype=torch.float16, device=DEV)

    def step():
        s.cache.append(k, v, b)
        s.cache.attention(q, b, out=out)
    b.lengths.zero_()                                          # (rows in front of the first token: nothing is written)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(2):
        have = [h + m for h, m in zip(have, news)]
        if any(h > n_ for h, n_ in zip(have, lens)):
            break
        b.lengths.copy_(ints(have))
        k.copy_(s.rows(s.k, have, news))
        v.copy_(s.rows(s.v, have, news))
        q.copy_(torch.cat([s.noise(m, 8) for m in news]))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device=DEV).sum().item()   # the allocator's memory in use by others between replays
        check_attention(s, have, news, out, None, q)
        assert torch.equal(out, s.cache.attention(q, b)) and np.isfinite(junk)


@pytest.mark.parametrize("starts", [[[0, 3, 8], [0, 6, 8], [2, 2, 8], [1, 7, 7], [0, 1, 2]], [[0, 40, 44], [0, 4, 44], [3, 3, 30], [0, 44, 44], [20, 21, 22]]],
                         ids=["few", "chunk"])
def test_captured_steps_follow_rows_and_pages(starts):
    """Between replays rows move from one sequence to the other and pages to other places of the pool."""
    lens = [900, 640]
    s = Setup(lens, hq=8, hkv=2, bits=8, page=16, seed=17)
    s.fill()
    n = max(x[2] for x in starts)
    b = R.RkvPagedBatch(s.dtable, ints(starts[0]), ints(lens), n_rows=n, max_new=max(max(x[1] - x[0], x[2] - x[1]) for x in starts), max_len=900)
    k, v = (torch.zeros(n, 2, 128, dtype=torch.float16, device=DEV) for _ in range(2))
    q, out = torch.zeros(n, 8, 128, dtype=torch.float16, device=DEV), torch.zeros(n, 8, 128, dtype=torch.float16, device=DEV)

    def step():
        s.cache.append(k, v, b)
        s.cache.attention(q, b, out=out)
    b.lengths.zero_()                                          # (rows in front of the first token: nothing is written)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, at in enumerate(starts):
        have = [900 - 7 * i, 640 - 100 * i]
        news = [at[1] - at[0], at[2] - at[1]]
        b.row_start.copy_(ints(at))
        b.lengths.copy_(ints(have))
        pages = s.cache.mem.view(s.n_pages, -1)                # every page moves on by one place
        pages.copy_(pages.roll(1, 0))
        used = s.dtable >= 0
        s.dtable[used] = (s.dtable[used] + 1) % s.n_pages
        k[at[0]:at[2]] = s.rows(s.k, have, news)
        v[at[0]:at[2]] = s.rows(s.v, have, news)
        q.copy_(s.noise(n, 8))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        junk = torch.randn(1 << 20, device=DEV).sum().item()
        check_attention(s, have, news, out, None, q, rows_from=at[0])
        assert torch.isnan(out[:at[0]]).all() and torch.isnan(out[at[2]:]).all()
        again = s.cache.attention(q, b)
        assert torch.equal(out[at[0]:at[2]], again[at[0]:at[2]]) and np.isfinite(junk)


def test_two_graphs_and_streams_at_once():
    """Captured calls that need work space, replayed on two streams at the same time."""
    lens, news = [6000], [1]
    sets = [Setup(lens, hq=8, hkv=1, seed=20 + i) for i in range(2)]
    graphs, outs, want, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    for s in sets:
        s.fill()
        q, b = s.noise(1, 8).to(DEV), s.batch(lens, news)
        want.append(s.cache.attention(q, b))
        out = torch.zeros_like(want[-1])
        s.keep = (q, b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(20):
                s.cache.attention(q, b, out=out)
        graphs.append(g)
        outs.append(out)
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_calls_on_another_stream():
    lens, news = [5000, 40], [1, 40]
    s = Setup(lens, hq=8, hkv=1, seed=30)
    s.fill()
    q, b = torch.cat([s.noise(m, 8) for m in news]).to(DEV), s.batch(lens, news)
    want = s.cache.attention(q, b)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        outs = [s.cache.attention(q, b) for _ in range(10)]
    torch.cuda.current_stream().wait_stream(st)
    assert all(torch.equal(o, want) for o in outs)


def test_no_rows():
    s = Setup([10], seed=1)
    s.fill()
    b = R.RkvPagedBatch(s.dtable, ints([0, 0]), ints([10]), n_rows=0)
    k, v = s.cache.read(b)
    s.cache.append(k, v, b)
    out, lse = s.cache.attention(torch.zeros(0, 4, 128, dtype=torch.float16, device=DEV), b, want_lse=True)
    assert k.shape == (0, 2, 128) and out.shape == (0, 4, 128) and lse.shape == (0, 4)


def test_refusals_of_the_binding():
    s = Setup([40], hq=4, hkv=2, seed=1)
    s.fill()
    b = s.batch([40], [8])
    x = torch.zeros(8, 2, 128, dtype=torch.float16, device=DEV)
    q = torch.zeros(8, 4, 128, dtype=torch.float16, device=DEV)
    for bad in (x.bfloat16(), x.cpu(), x.float(), None):
        with pytest.raises(TypeError):
            s.cache.append(bad, x, b)
    for bad in (x[:7], x[:, :1], x[..., :64], x.transpose(1, 2).contiguous().transpose(1, 2), torch.zeros(8, 2, 256, dtype=torch.float16, device=DEV)[..., ::2]):
        with pytest.raises(ValueError):
            s.cache.append(x, bad, b)
    with pytest.raises(ValueError):
        s.cache.attention(x, b)
    with pytest.raises(R.RkvError):                            # rows that lie on top of each other
        s.cache.append(x[:1].expand(8, 2, 128), x, b)
    with pytest.raises(R.RkvError):                            # not aligned
        s.cache.append(torch.zeros(8 * 256 + 1, dtype=torch.float16, device=DEV)[1:].view(8, 2, 128), x, b)
    for kw in (dict(scale=float("nan")), dict(scale=1e300)):
        with pytest.raises(R.RkvError):
            s.cache.attention(q, b, **kw)
    for kw in (dict(out=q.float()), dict(lse=q)):
        with pytest.raises(TypeError):
            s.cache.attention(q, b, **kw)
    for kw in (dict(out=q[:4]), dict(lse=torch.zeros(8, 2, device=DEV)), dict(window=-1), dict(window=2**32)):
        with pytest.raises(ValueError):
            s.cache.attention(q, b, **kw)
    with pytest.raises(ValueError):
        R.RkvPagedCache(s.cfg, device=DEV, mem=torch.zeros(100, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        R.RkvPagedBatch(s.dtable, ints([0, 1, 2]), ints([40]), 2)
    for kw in (dict(n_rows=2**32 + 8), dict(n_rows=8, max_new=2**32 + 8), dict(n_rows=8, max_len=2**32 + 40)):   # (cut to 32 bits they would do)
        with pytest.raises(ValueError):
            R.RkvPagedBatch(s.dtable, ints([0, 8]), ints([40]), **kw)
    with pytest.raises(R.RkvError):
        s.cache.attention(q, R.RkvPagedBatch(s.dtable, ints([0, 8]), ints([40]), 8, max_len=10**6))
    # too little work space is refused by the library, before anything runs
    import ctypes as C
    big = s.batch([40], [8]).to_c(s.cfg)
    need = C.c_size_t()
    c = s.cfg.to_c()
    assert s.cache.lib.rkv_paged_scratch(C.byref(c), C.byref(big), C.byref(need)) == B.RKV_OK
    if need.value:
        rc = s.cache.lib.rkv_paged_attention(C.byref(c), s.cache.mem.data_ptr(), C.byref(big), q.data_ptr(), 512, 1, 0, 0.1, q.data_ptr(), None,
                                             None, 0, None)
        assert rc == B.RKV_EINVAL
