"""The cache in pages without a GPU: its oracle against closed forms, the sizes, and every refusal of the calls (all
of them come before anything is launched)."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import paper_2501_16383_amd as R
from oracle import paged_oracle as O
from paper_2501_16383_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(R.library_path()):
        from paper_2501_16383_amd.build import build_library
        build_library()
    return R.load_library()


# ---- the oracle ----

def test_grids_are_the_formats():
    bits = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.E4M3, bits) and O.E4M3[-1] == 448 and O.E2M1[-1] == 6


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_stored_numbers_of_eight_bits_by_another_conversion(dtype):
    """Scales that need no search: blocks whose largest magnitude is a power of two.  Codes by torch's conversion."""
    t = torch.float16 if dtype == "fp16" else torch.bfloat16
    x = (torch.rand(200, 64, generator=torch.Generator().manual_seed(3)) * 2 - 1).to(t)
    x[:, ::32] = 1.0
    two = 2.0 ** -8                                            # 1 = 256 * 2^-8 <= 448 * 2^-8, and 448 * 2^-9 < 1
    want = (x.float() / two).to(torch.float8_e4m3fn).double() * two
    assert np.array_equal(O.stored(x.double().numpy(), 8, dtype), want.numpy())
    assert np.array_equal(O.scales(x.double().numpy(), 8, dtype), np.full((200, 2), -8.0))


@pytest.mark.parametrize("bits,dtype", [(b, d) for b in (8, 4) for d in ("fp16", "bf16")])
def test_stored_numbers_are_of_the_type_and_near(bits, dtype):
    """Every stored number is one of the type; the error is at most half the grid's step: 2^-4 (8 bits) of the number or
    2^-2 (4 bits), or half the smallest step, or what the cap of the largest numbers takes off."""
    t = torch.float16 if dtype == "fp16" else torch.bfloat16
    allbits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(t)
    x = allbits[torch.isfinite(allbits)].sort().values.repeat_interleave(32).double().numpy().reshape(-1, 32)   # a block of each
    x[:, 1:] *= np.linspace(1, 0.01, 31)
    x = torch.from_numpy(x).to(t).double().numpy()
    s = O.stored(x, bits, dtype)
    assert np.array_equal(torch.from_numpy(s).to(t).double().numpy(), s)
    grid, low, top = O.limits(bits, dtype)
    two = np.exp2(O.scales(x, bits, dtype))
    half = np.maximum(np.abs(x) * 2.0 ** (-4 if bits == 8 else -2), two * grid[1] / 2)
    assert (np.abs(s - x) <= np.maximum(half, np.abs(x) - top)).all()
    assert (np.abs(x).max(-1) <= grid[-1] * two[:, 0]).all() or np.abs(x).max() > top
    small = (two[:, 0] > 2.0**low)                             # no smaller scale would do
    assert (np.abs(x[small]).max(-1) > grid[-1] * two[small, 0] / 2).all()


def test_stored_block_that_is_not_finite():
    x = np.ones((3, 64))
    x[0, 5], x[1, 40] = np.nan, -np.inf
    s = O.stored(x, 8, "fp16")
    assert np.isnan(s[0, :32]).all() and np.isnan(s[1, 32:]).all() and (s[2] == 1).all() and (s[0, 32:] == 1).all()


def test_attention_oracle_by_closed_forms():
    rng = np.random.default_rng(0)
    k, v, q = rng.normal(size=(9, 2, 64)), rng.normal(size=(9, 2, 64)), rng.normal(size=(9, 4, 64))
    out, lse, *_ = O.attention(np.zeros_like(q), k, v, 0)      # no scores: running means
    mean = np.cumsum(v, 0) / np.arange(1, 10)[:, None, None]
    assert np.allclose(out, np.repeat(mean, 2, axis=1)) and np.allclose(lse, np.log(np.arange(1, 10))[:, None])
    out, _, *_ = O.attention(q, k, v, 0, window=1)             # each row sees itself
    assert np.allclose(out, np.repeat(v, 2, axis=1))
    out, lse, *_ = O.attention(q, k, v, -2)                    # two rows in front of the first token
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all() and np.isfinite(lse[2:]).all()
    ref = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q).transpose(0, 1), torch.from_numpy(np.repeat(k, 2, 1)).transpose(0, 1),
        torch.from_numpy(np.repeat(v, 2, 1)).transpose(0, 1)).transpose(0, 1).numpy()
    assert np.allclose(O.attention(q, k, v, 0, causal=False)[0], ref)


# ---- sizes and refusals ----

def test_sizes(lib):
    for bits, per_row in ((16, 512), (8, 264), (4, 136)):
        assert R.paged_sizes(R.RkvPagedConfig(32, 8, 100, bits=bits, page_tokens=32)) == 100 * 8 * 32 * per_row
    assert R.paged_sizes(R.RkvPagedConfig(1, 1, 1, head_dim=64, bits=4, page_tokens=16)) == 16 * 68
    assert R.paged_sizes(R.RkvPagedConfig(32, 8, 2**31 - 1)) == (2**31 - 1) * 8 * 64 * 264


@pytest.mark.parametrize("field,value", [("n_q_heads", 33), ("n_q_heads", 0), ("n_kv_heads", 0), ("n_kv_heads", 257), ("n_pages", 0),
                                         ("head_dim", 96), ("head_dim", 256), ("page_tokens", 8), ("page_tokens", 48), ("page_tokens", 512),
                                         ("bits", 2), ("bits", 32), ("dtype", 2), ("dtype", -1)])
def test_configurations_that_are_refused(lib, field, value):
    cfg = R.RkvPagedConfig(32, 8, 100)
    setattr(cfg, field, value)
    with pytest.raises(R.RkvError) as e:
        R.paged_sizes(cfg)
    assert e.value.code == B.RKV_EINVAL


FAKE = 1 << 20                                                 # an address that nothing may look at


def calls(lib, cfg=None, batch=None, pool=FAKE, k=FAKE, v=FAKE, ks=1024, vs=1024, q=FAKE, qs=4096, causal=1, window=0, scale=0.1, out=FAKE,
          lse=None, scratch=FAKE, scratch_bytes=1 << 40):
    """Return codes of append, read and attention."""
    c = (cfg or R.RkvPagedConfig(32, 8, 100)).to_c()
    b = C.byref(batch) if batch is not None else None
    return [lib.rkv_paged_append(C.byref(c), pool, b, k, ks, v, vs, None), lib.rkv_paged_read(C.byref(c), pool, b, k, ks, v, vs, None),
            lib.rkv_paged_attention(C.byref(c), pool, b, q, qs, causal, window, scale, out, lse, scratch, scratch_bytes, None)]


def a_batch(**kw):
    f = dict(dev_page_table=FAKE, dev_row_start=FAKE, dev_lengths=FAKE, n_seqs=4, max_pages=10, n_rows=7, max_new=4, max_len=640)
    f.update(kw)
    return B._CPagedBatch(**f)


@pytest.mark.parametrize("kw", [dict(dev_page_table=None), dict(dev_row_start=None), dict(dev_lengths=None), dict(dev_lengths=FAKE + 2), dict(n_seqs=0),
                                dict(n_seqs=65537), dict(max_pages=0), dict(n_rows=-1), dict(max_new=0), dict(max_new=8), dict(max_len=0),
                                dict(max_len=641), dict(n_rows=1 << 26, max_pages=1 << 30)], ids=str)
def test_batches_that_are_refused(lib, kw):
    batch = a_batch(**kw)
    assert calls(lib, batch=batch) == [B.RKV_EINVAL] * 3
    c = R.RkvPagedConfig(32, 8, 100).to_c()
    assert lib.rkv_paged_scratch(C.byref(c), C.byref(batch), None) == B.RKV_EINVAL


def test_arguments_that_are_refused(lib):
    E = B.RKV_EINVAL
    assert calls(lib) == [E] * 3                               # no batch
    b = a_batch()
    assert calls(lib, R.RkvPagedConfig(32, 8, 0), b) == [E] * 3
    for bad in (None, FAKE + 8):
        assert calls(lib, batch=b, pool=bad) == [E] * 3
        assert calls(lib, batch=b, k=bad, q=bad) == [E] * 3
        assert calls(lib, batch=b, v=bad, out=bad) == [E] * 3
    for stride in (1016, 1020, 0, -1024, 1 << 31):             # shorter than a row, not of eight elements, backwards, too long
        assert calls(lib, batch=b, ks=stride)[:2] == [E] * 2 and calls(lib, batch=b, vs=stride)[:2] == [E] * 2
    for stride in (4088, 4100, 0, -4096, 1 << 31):
        assert calls(lib, batch=b, qs=stride)[2] == E
    for kw in (dict(causal=2), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(lse=FAKE + 2)):
        assert calls(lib, batch=b, **kw)[2] == E


@pytest.mark.parametrize("max_new,n_seqs", [(1, 4), (9, 1), (4, 4), (200, 1), (200, 4)])
@pytest.mark.parametrize("D,bits", [(128, 16), (64, 4)])
def test_work_space_that_is_refused(lib, max_new, n_seqs, D, bits):
    """Batches that are cut into splits: without the work space, with one that is not aligned or a byte short nothing is launched."""
    cfg = R.RkvPagedConfig(8, 2, 400, head_dim=D, bits=bits)
    batch = a_batch(n_seqs=n_seqs, n_rows=max_new + 3, max_new=max_new, max_pages=100, max_len=6000)
    need, c = C.c_size_t(), cfg.to_c()
    assert lib.rkv_paged_scratch(C.byref(c), C.byref(batch), C.byref(need)) == B.RKV_OK and need.value > 1 << 16
    for kw in (dict(scratch=None, scratch_bytes=need.value), dict(scratch=FAKE + 16, scratch_bytes=need.value), dict(scratch=FAKE + 128, scratch_bytes=1 << 40),
               dict(scratch_bytes=need.value - 1), dict(scratch_bytes=0)):
        assert calls(lib, cfg, batch, qs=8 * D, **kw)[2] == B.RKV_EINVAL


@pytest.mark.parametrize("D", [64, 128])
def test_batches_that_no_launch_holds(lib, D):
    """2^32 threads and more: one for eight channels of a row in append and read, 512 for a tile of columns in attention."""
    cfg, E = R.RkvPagedConfig(256, 256, 100, head_dim=D), 256 * D
    rows = 2**35 // E                                          # rows * heads * D = 2^35
    batch = a_batch(n_rows=rows, max_new=1)
    assert calls(lib, cfg, batch, ks=E, vs=E, qs=8)[:2] == [B.RKV_EINVAL] * 2
    batch = a_batch(n_rows=2**22, n_seqs=65535, max_new=100)   # (2^22 * 256 / 256 + 65535 * 256) workgroups of 512
    assert calls(lib, cfg, batch, ks=8, vs=8, qs=E)[2] == B.RKV_EINVAL
    n, c = C.c_size_t(77), cfg.to_c()
    assert lib.rkv_paged_scratch(C.byref(c), C.byref(batch), C.byref(n)) == B.RKV_EINVAL and n.value == 77
    batch.max_new = 32                                         # few rows: a workgroup for a sequence and head
    assert lib.rkv_paged_scratch(C.byref(c), C.byref(batch), C.byref(n)) == B.RKV_OK


def test_no_rows_is_nothing_to_do(lib):
    b = a_batch(n_rows=0, max_new=0, dev_page_table=None)
    assert calls(lib, batch=b, pool=None, k=None, v=None, q=None, out=None, scratch=None, scratch_bytes=0) == [B.RKV_OK] * 3
    n, c = C.c_size_t(77), R.RkvPagedConfig(32, 8, 100).to_c()
    assert lib.rkv_paged_scratch(C.byref(c), C.byref(b), C.byref(n)) == B.RKV_OK and n.value == 0


def test_null_arguments(lib):
    assert lib.rkv_paged_sizes(None, None) == B.RKV_EINVAL
    assert lib.rkv_paged_append(None, None, None, None, 0, None, 0, None) == B.RKV_EINVAL
    assert lib.rkv_paged_read(None, None, None, None, 0, None, 0, None) == B.RKV_EINVAL
    assert lib.rkv_paged_scratch(None, None, None) == B.RKV_EINVAL
    assert lib.rkv_paged_attention(None, None, None, None, 0, 1, 0, 1.0, None, None, None, 0, None) == B.RKV_EINVAL


def test_the_binding_wants_device_tensors():
    x = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(TypeError):
        R.RkvPagedBatch(torch.zeros(2, 4, dtype=torch.int32), x, x[:2], 1)
    with pytest.raises(TypeError):
        R.RkvPagedBatch(None, x, x[:2], 1)
