"""The 4-bit cache's calls on addresses that only the C interface takes (rows, queries and outputs on
16-byte boundaries), on further page sizes, and the alignment of their workspaces."""
import numpy as np
import pytest
import torch

from paper_2608_18486_gb300 import _lib as W
from paper_2608_18486_gb300.session import DecodeSession, Q4Cache
from tests import _q4 as Q
from tests import test_q4_gpu as base
from tests.test_q4_gpu_rows import FORMS, case, config, form

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", base.KINDS)
@pytest.mark.parametrize("page", [4, 32, 128])
def test_write_holds_the_nearest_values_in_pages_of(page, dtype, d):
    base.test_write_holds_the_nearest_values(dtype, d, page)


@pytest.mark.parametrize("dtype,d", base.KINDS)
@pytest.mark.parametrize("page", [4, 16])
@pytest.mark.parametrize("at", [(16, 0), (0, 16), (16, 48)])
def test_copies_of_rows_on_16_byte_boundaries(dtype, d, page, at):
    """The same bytes as from rows on 32-byte boundaries, and nothing beside them."""
    rng = np.random.default_rng(d)
    k, Hkv, B, maxp = 2, 3, 2, 96 // page
    pages, tdt = B * maxp, torch.float32 if dtype == "f32" else torch.bfloat16
    cfg = W.make_config(k, k, 64, Hkv, Hkv, d, 1, page, dtype, [0, 1])
    s, want, got = DecodeSession(cfg, B, pages, maxp), Q4Cache(cfg, pages), Q4Cache(cfg, pages)
    rows = base.special_rows(rng, 2 * s.k_pool.numel() // d, d, dtype).reshape(2, *s.k_pool.shape)
    for pool, x in zip((s.k_pool, s.v_pool), rows):
        pool.copy_(torch.from_numpy(x).to(tdt))
    size = s.k_pool.numel() * s.k_pool.element_size()
    bufs = [torch.full((size + 256,), 0x3C, dtype=torch.uint8, device="cuda") for _ in range(2)]
    near = [b[o:o + size].view(tdt).view(s.k_pool.shape) for b, o in zip(bufs, at)]
    cache = W.wm_cache_alloc(cfg, s.cache_buf, s.cache_buf.numel(), pages)
    cache.k_pool, cache.v_pool = (x.data_ptr() for x in near)
    for x, pool in zip(near, (s.k_pool, s.v_pool)):
        x.copy_(pool)
    dev = [torch.from_numpy(rng.permutation(pages).reshape(B, maxp).astype(np.int32)).cuda() for _ in range(2)]
    first, last = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([3, 17], [91, 96]))
    for q4 in (want, got):
        q4.cache_buf.fill_(0x5A)
    stream = torch.cuda.current_stream().cuda_stream
    s.q4_write(want, *dev, first, last, span=96)
    assert W.wm_q4_write(cfg, cache, dev[0], got.cache, dev[1], first, last, 96, B, maxp, s.status, stream) == W.WM_OK
    assert torch.equal(want.cache_buf, got.cache_buf)
    for x in (*near, s.k_pool, s.v_pool):
        x.fill_(5)
    s.q4_read(want, dev[1], dev[0], first, last, span=96)
    assert W.wm_q4_read(cfg, got.cache, dev[1], cache, dev[0], first, last, 96, B, maxp, s.status, stream) == W.WM_OK
    for x, pool, b, o in zip(near, (s.k_pool, s.v_pool), bufs, at):
        assert torch.equal(x.view(torch.uint8), pool.view(torch.uint8))
        assert bool((b[:o] == 0x3C).all()) and bool((b[o + size:] == 0x3C).all())
    assert s.read_status() == 0


def between(x):
    """The tensor on a 16-byte boundary that is no 32-byte one."""
    n = x.numel() * x.element_size()
    y = torch.full((n + 64,), 0x3C, dtype=torch.uint8, device="cuda")[16:16 + n].view(x.dtype).view(x.shape)
    assert y.data_ptr() % 32 == 16
    return y.copy_(x)


@pytest.mark.parametrize("f", [FORMS[0], FORMS[2], FORMS[5], FORMS[6], (4, 3, [90, 70], 2, 64, 16, 8, None)])
def test_rows_and_outputs_on_16_byte_boundaries(f):
    G, Tq, lens, Hkv, d, page, maxp, cut = f
    x = Q.Q4(lens, Hkv=Hkv, G=G, d=d, page=page, k=1, max_pages=maxp) if cut is None else case(*f)
    s, q4 = x.session(), x.q4()
    table, n = x.q4_dev()
    pos = torch.from_numpy(np.stack([np.arange(n - Tq, n) for n in x.lens]).astype(np.int32)).cuda()
    q = x.queries(x.B, Tq).cuda()
    want = torch.empty_like(q)
    got = between(torch.zeros_like(q))
    s.q4_rows_attn(0, q, pos, q4, table, want)
    s.q4_rows_attn(0, between(q), pos, q4, table, got)
    assert torch.equal(got, want)
    one = q[:, 0].contiguous()
    want, got = torch.empty_like(one), between(torch.zeros_like(one))
    s.q4_decode_attn(0, one, q4, table, n, want)
    s.q4_decode_attn(0, between(one), q4, table, n, got)
    assert torch.equal(got, want) and s.read_status() == 0


def test_workspaces_are_multiples_of_256_bytes():
    seen = set()
    for B in (1, 3, 7, 64):
        for maxp in (1, 5, 64, 1023, 8192):
            for Hq, Hkv, d in ((6, 3, 96), (32, 8, 128), (12, 12, 64), (8, 1, 128)):
                c = config(Hq, Hkv, d, 16)
                n = W.wm_q4_decode_attn_workspace(c, B, maxp)
                assert n > 0 and n % 256 == 0
                seen.add("clusters" if n == 256 else "spread")
                for Tq in (1, 2, 61, 300):
                    n = W.wm_q4_rows_attn_workspace(c, B, Tq, maxp)
                    assert n > 0 and n % 256 == 0
                    at = form(c, B, Tq, maxp) if n > 10 ** 8 else None
                    seen.add("cut" if at and at[1] else "whole" if at else "few")
    assert seen == {"clusters", "spread", "cut", "whole", "few"}
