"""The quantised cache's definition, and refusals of the calls that serve chunks and quantised caches (no GPU)."""
import numpy as np
import pytest

import paper_2608_23463_gb300 as pf
from oracle import local as OL
from tests.test_local_host import A, cache, lib, paged, qk, refused, rows  # noqa: F401


def test_definition():
    """Whole numbers and exponents by going through all exponents."""
    rng = np.random.default_rng(1)
    y = rng.standard_normal((200, 16)) * np.exp2(rng.integers(-140, 100, (200, 1)))
    y[0], y[1], y[2, 3] = 0.0, 127.0, 127.0 + 2.0 ** -40
    x, e = OL.quantise(y)
    for r in range(200):
        least = next(k for k in range(-126, 105) if np.abs(y[r]).max() <= 127 * 2.0 ** k)
        assert e[r] == least
        assert (x[r] == np.round(y[r] / 2.0 ** least)).all() and np.abs(x[r]).max() <= 127
    v = OL.values(x, e)
    assert (np.abs(v - y) <= 2.0 ** e.astype(float)[:, None] / 2).all()
    # bf16 holds them: the upper 16 of fp32's bits
    f = v.astype(np.float32)
    assert (f == v).all() and not (f.view(np.uint32) & 0xffff).any()
    x, e = OL.quantise(np.array([[1.0, np.inf], [np.nan, 0.0], [127.1 * 2.0 ** 104, 0.0], [127 * 2.0 ** 104, 0.0]]))
    assert e.tolist() == [-128, -128, -128, 104] and np.isnan(OL.values(x, e)[:3]).all()


def test_chunk_of_one_is_the_newest_token():
    rng = np.random.default_rng(2)
    K, V = rng.standard_normal((2, 9, 2, 16, 8))
    table, length = rng.permutation(9).reshape(3, 3), [40, 1, 17]
    q = rng.standard_normal((3, 4, 8))
    for w, s in ((0, 0), (7, 3)):
        a, b = OL.paged_attn(q, K, V, table, length, w, s), OL.paged_chunk(q, K, V, table, length, [0, 1, 2, 3], w, s)
        for x, y in zip(a, b):  # float64 sums of 40 terms in another order
            np.testing.assert_allclose(x, y, rtol=1e-12, atol=1e-13)


def exp(K=A, V=A):
    return pf.PagedExp(K, V)


def test_refusals():
    bad, no = pf.PF_ERR_INVALID_ARG, pf.PF_ERR_UNSUPPORTED
    B = 1 << 20
    chunk = lambda d=paged(), n=8, q=A, ld=256, start=A, c=cache(), e=None, out=B, ld_o=256, ws=A, size=1 << 30: \
        pf.pf_paged_chunk_attn(d, n, q, ld, start, c, e, out, ld_o, ws, size)
    read = lambda d=paged(), n=8, start=A, c=cache(), e=None, k=A, ld_k=128, v=B, ld_v=128: \
        pf.pf_paged_read(d, n, start, c, e, k, ld_k, v, ld_v)
    attn = lambda d=paged(), q=A, ld=256, c=cache(), e=exp(), out=A, ld_o=256, ws=A, size=1 << 30: \
        pf.pf_paged_attn_q8(d, q, ld, c, e, out, ld_o, ws, size)
    app = lambda d=paged(), k=qk(), n=3, x=rows(), start=None, c=cache(), e=exp(), qo=A, ld=256: \
        pf.pf_paged_append_q8(d, k, n, x, A, A, start, None, c, e, qo, ld)
    for s, kws in ((bad, (dict(batch=0), dict(n_kv=3), dict(page=0), dict(page=24), dict(max_pages=0), dict(n_pages=0),
                          dict(window=-1), dict(n_sink=-1))),
                   (no, (dict(batch=2049), dict(dh=80), dict(n_heads=34)))):
        for kw in kws:
            for f in (chunk, read, attn, app):
                refused(s, f, paged(**kw))
            assert pf.pf_paged_chunk_workspace_size(paged(**kw), 8) == 0
    for kw in (dict(K=None), dict(V=A + 2), dict(table=None), dict(length=None)):
        for f in (chunk, read, attn, app):
            refused(bad, lambda: f(c=cache(**kw)))
    for e in (exp(K=None), exp(V=None), exp(K=A + 8), exp(V=A + 1)):
        for f in (chunk, read, attn, app):
            refused(bad, lambda: f(e=e))
    refused(bad, lambda: attn(e=None))
    refused(bad, lambda: app(e=None))
    for kw in (dict(n=-1), dict(n=1 << 31), dict(start=None), dict(q=None), dict(q=A + 8), dict(ld=252), dict(ld=248),
               dict(out=None), dict(ld_o=128), dict(out=A), dict(out=A + 64), dict(out=A + 512 * 7)):
        refused(bad, lambda: chunk(**kw))
    for kw in (dict(n=-1), dict(start=None), dict(k=None), dict(v=B + 2), dict(ld_k=64), dict(ld_v=132), dict(v=A),
               dict(k=B + 256 * 7)):
        refused(bad, lambda: read(**kw))
    need = pf.pf_paged_chunk_workspace_size(paged(max_pages=100), 8)
    assert need > 0
    for kw in (dict(size=need - 1), dict(ws=None), dict(ws=A + 4)):
        refused(pf.PF_ERR_WORKSPACE, lambda: chunk(paged(max_pages=100), **kw))
    assert chunk(n=0, q=0, out=0) is None and read(n=0, k=0, v=0) is None  # no token: nothing to do
    refused(no, lambda: app(k=qk(dtype=pf.PF_F32)))
    refused(bad, lambda: app(n=4))


def test_chunk_workspace_stays_small():
    """Two places of an item's rows for each of 152 CTAs at most, whatever the cache and the call hold."""
    size = pf.pf_paged_chunk_workspace_size
    top = 153 * 16 + 256 + 304 * 256 * (8 + 128 * 4)
    for d, n in ((paged(batch=2048, max_pages=1 << 30, dh=128), 1 << 24), (paged(max_pages=1 << 30, n_heads=32, dh=128), 5000)):
        assert 0 < size(d, n) <= top + 512
    assert size(paged(batch=1, n_heads=1, n_kv=1, max_pages=1 << 20), 3) <= top // 3
    assert size(paged(max_pages=8), 100) == 0 and size(paged(), 0) == 0


def test_newest_token_workspace():
    """Of a quantised cache: what the call needs is what it takes, and a broken description has none."""
    size = pf.pf_paged_attn_q8_workspace_size
    d = paged(max_pages=1 << 20)
    need = size(d)
    assert need > 0
    attn = lambda ws, n: pf.pf_paged_attn_q8(d, A, 256, cache(), exp(), A, 256, ws, n)
    for ws, n in ((A, need - 1), (None, need), (A + 8, need)):
        refused(pf.PF_ERR_WORKSPACE, lambda: attn(ws, n))
    for kw in (dict(batch=0), dict(batch=2049), dict(dh=80), dict(page=24)):
        assert size(paged(**kw)) == 0


def test_python_refusals():
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace

    from paper_2608_23463_gb300 import local
    bad = pf.PF_ERR_INVALID_ARG
    mk = lambda **kw: local.PagedKVCache(1, 4, 2, 64, 16, 4, 2, device="cpu", **kw)
    i8, shape = torch.int8, (4, 2, 16)
    e, K = torch.zeros(shape, dtype=i8), torch.zeros(shape + (64,), dtype=i8)
    for kw in (dict(dtype=torch.float16), dict(dtype=i8), dict(K_exp=e), dict(dtype=i8, K_exp=e.float()), dict(K=K),
               dict(dtype=i8, K=K.bfloat16()), dict(dtype=i8, V_exp=e[:, :, :8]), dict(dtype=i8, V_exp=e.mT)):
        refused(bad, lambda: mk(**kw))
    c = local.PagedKVCache.__new__(local.PagedKVCache)
    c.batch, c.len = 2, SimpleNamespace(device=torch.device("cuda", 1))
    c.at = c.at_cache = c.at_exp = 0
    c.desc, c.cache = paged(), cache()
    from ctypes import addressof
    c.at, c.at_cache = addressof(c.desc), addressof(c.cache)
    refused(bad, lambda: c.read(torch.zeros(3, dtype=torch.int32)))  # rows are not known
    q = torch.zeros(8, 256, dtype=torch.bfloat16)
    for x in (q, q.float(), None, 7):
        refused(bad, lambda: c.attend(x, start=torch.zeros(4, dtype=torch.int32)))
