"""Argument checks of the local stream's operators (no GPU): every refusal comes
before anything is launched."""
import pytest

import paper_2608_23463_gb300 as pf


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2608_23463_gb300.buildlib import build
    build()
    return pf.load()


A = 1 << 12  # an aligned address that nothing reads


def refused(status, f, *a):
    with pytest.raises(pf.ProxyFormerError) as e:
        f(*a)
    assert e.value.status == status, e.value


def qk(n_heads=4, n_kv=2, dh=64, dtype=pf.PF_BF16, n_axes=1, pairs=(32, 0, 0), theta=1e4, eps=1e-6):
    return pf.QKDesc(n_heads, n_kv, dh, dtype, n_axes, pairs, theta, eps)


def rows(q=A, k=A, v=A, ld_q=256, ld_k=128, ld_v=128):
    return pf.QKV(q, k, v, ld_q, ld_k, ld_v)


def test_rope_refusals():
    f = lambda d=qk(), n=8, L=8, x=rows(), pos=None, out=rows(): pf.pf_qk_rope_fwd(d, n, L, x, A, A, pos, out)
    bad, no = pf.PF_ERR_INVALID_ARG, pf.PF_ERR_UNSUPPORTED
    for kw in (dict(n_heads=5), dict(n_kv=0), dict(n_heads=-4), dict(dtype=7), dict(n_axes=4), dict(n_axes=-1),
               dict(pairs=(33, 0, 0)), dict(n_axes=2, pairs=(30, 3, 0)), dict(pairs=(-1, 0, 0)), dict(theta=0.0),
               dict(theta=float("nan")), dict(eps=0.0)):
        refused(bad, f, qk(**kw))
        assert pf.pf_qk_rope_workspace_size(qk(**kw)) == 0
    refused(no, f, qk(dh=96))
    refused(bad, lambda: f(n=-1))
    refused(bad, lambda: f(n=1 << 31))
    refused(bad, lambda: f(L=0))
    refused(bad, lambda: f(qk(n_axes=2, pairs=(16, 16, 0))))  # several axes need positions
    for kw in (dict(q=None), dict(k=A + 8), dict(ld_q=248), dict(ld_k=132), dict(ld_q=1 << 40)):
        refused(bad, lambda: f(x=rows(**kw)))
        refused(bad, lambda: f(out=rows(**kw)))
    refused(bad, lambda: f(qk(dtype=pf.PF_F32), x=rows(ld_q=258)))


def test_rope_backward_refusals():
    def f(d=qk(), n=8, dout=rows(), dx=rows(), w_q=A, dw_q=A, ws=A, size=1 << 30):
        pf.pf_qk_rope_bwd(d, n, 8, rows(), w_q, A, None, dout, dx, dw_q, A, ws, size)
    refused(pf.PF_ERR_INVALID_ARG, lambda: f(dout=rows(q=None)))
    refused(pf.PF_ERR_INVALID_ARG, lambda: f(dx=rows(ld_k=64)))
    refused(pf.PF_ERR_INVALID_ARG, lambda: f(w_q=None))
    need = pf.pf_qk_rope_workspace_size(qk())
    refused(pf.PF_ERR_WORKSPACE, lambda: f(size=need - 1))
    refused(pf.PF_ERR_WORKSPACE, lambda: f(ws=None))
    refused(pf.PF_ERR_WORKSPACE, lambda: f(ws=A + 4))


def win(batch=2, L=300, n_heads=4, n_kv=2, dh=64, window=100, n_sink=4):
    return pf.WindowDesc(batch, L, n_heads, n_kv, dh, window, n_sink)


def test_window_refusals():
    bad, no = pf.PF_ERR_INVALID_ARG, pf.PF_ERR_UNSUPPORTED
    B = A * 2  # addresses of the gradients
    grads = lambda **kw: rows(**{**dict(q=B, k=B, v=B), **kw})
    fwd = lambda d=win(), x=rows(), out=A, ld=256, saved=A: pf.pf_window_attn_fwd(d, x, out, ld, saved)

    def bwd(d=win(), x=rows(), out=A, ld=256, saved=A, dout=A, ld_d=256, dx=None, ws=A, size=1 << 40):
        pf.pf_window_attn_bwd(d, x, out, ld, saved, dout, ld_d, dx or grads(), ws, size)
    for s, kws in ((bad, (dict(batch=0), dict(L=0), dict(n_kv=3), dict(window=-1), dict(n_sink=-2))),
                   (no, (dict(dh=128), dict(dh=32), dict(L=1 << 30), dict(batch=1 << 16, L=1 << 15),
                         dict(batch=1 << 20, L=1024, n_heads=64)))):
        for kw in kws:
            refused(s, fwd, win(**kw))
            refused(s, bwd, win(**kw))
            assert pf.pf_window_attn_workspace_size(win(**kw)) == pf.pf_window_attn_saved_size(win(**kw)) == 0
    for kw in (dict(q=None), dict(k=A + 8), dict(v=None), dict(ld_q=248), dict(ld_k=132), dict(ld_v=64)):
        refused(bad, lambda: fwd(x=rows(**kw)))
        refused(bad, lambda: bwd(x=rows(**kw)))
        refused(bad, lambda: bwd(dx=grads(**{n: (v + A if v and v > A else v) for n, v in kw.items()})))
    for kw in (dict(out=None), dict(out=A + 2), dict(ld=128), dict(ld=260)):
        refused(bad, lambda: fwd(**kw))
        refused(bad, lambda: bwd(**kw))
    refused(bad, lambda: bwd(saved=None))
    refused(bad, lambda: bwd(saved=A + 4))
    refused(bad, lambda: fwd(saved=A + 4))
    refused(bad, lambda: bwd(dout=None))
    refused(bad, lambda: bwd(dx=grads(k=A)))  # a gradient over an input
    need = pf.pf_window_attn_workspace_size(win())
    refused(pf.PF_ERR_WORKSPACE, lambda: bwd(size=need - 1))
    refused(pf.PF_ERR_WORKSPACE, lambda: bwd(ws=None))


def test_window_workspace_stays_small():
    """36 bytes of every row and head, and the sums of cut tiles: at most some thousands of 64 KB, whatever the length."""
    for d in (win(1, 262144, 16, 16, window=1024, n_sink=4), win(1, 262144, 16, 1, window=0),
              win(4, 65536, 32, 2, window=4096, n_sink=300), win(1, 1, 1, 1), win(3, 999, 64, 1, window=1, n_sink=998)):
        rest = 36 * d.batch * d.n_heads * d.L + 768
        heads, tiles = d.batch * d.n_kv, -(-d.L // 128)
        pieces = (pf.pf_window_attn_workspace_size(d) - rest) / 65536
        assert pieces <= 16 * 152 + 3 * heads + (304 + heads * tiles if heads * tiles < 152 else 0)


def paged(batch=3, n_heads=4, n_kv=2, dh=64, page=16, max_pages=4, n_pages=9, window=0, n_sink=0):
    return pf.PagedDesc(batch, n_heads, n_kv, dh, page, max_pages, n_pages, window, n_sink)


def cache(K=A, V=A, table=A, length=A):
    return pf.PagedCache(K, V, table, length)


def test_paged_refusals():
    bad, no = pf.PF_ERR_INVALID_ARG, pf.PF_ERR_UNSUPPORTED
    attn = lambda d=paged(), q=A, ld=256, c=cache(), out=A, ld_o=256, ws=A, size=1 << 30: pf.pf_paged_attn(
        d, q, ld, c, out, ld_o, ws, size)
    app = lambda d=paged(), k=qk(), n=3, x=rows(), start=None, c=cache(), qo=A, ld=256: pf.pf_paged_append(
        d, k, n, x, A, A, start, None, c, qo, ld)
    for s, kws in ((bad, (dict(batch=0), dict(n_kv=3), dict(page=0), dict(page=24), dict(max_pages=0), dict(n_pages=0),
                          dict(window=-1), dict(n_sink=-1))),
                   (no, (dict(batch=2049), dict(dh=80), dict(n_heads=34)))):
        for kw in kws:
            refused(s, attn, paged(**kw))
            refused(s, app, paged(**kw))
            refused(s, pf.pf_paged_advance, paged(**kw), None, cache())
            assert pf.pf_paged_attn_workspace_size(paged(**kw)) == 0
    for kw in (dict(K=None), dict(V=A + 2), dict(table=None), dict(length=None)):
        refused(bad, lambda: attn(c=cache(**kw)))
        refused(bad, lambda: app(c=cache(**kw)))
    refused(bad, lambda: pf.pf_paged_advance(paged(), None, cache(length=None)))
    for kw in (dict(q=None), dict(q=A + 8), dict(ld=252), dict(ld=248), dict(out=None), dict(ld_o=128)):
        refused(bad, lambda: attn(**kw))
    need = pf.pf_paged_attn_workspace_size(paged())
    refused(pf.PF_ERR_WORKSPACE, lambda: attn(size=need - 1))
    refused(pf.PF_ERR_WORKSPACE, lambda: attn(ws=None))
    refused(bad, lambda: app(k=qk(n_heads=8)))
    refused(bad, lambda: app(k=qk(dh=128)))
    refused(no, lambda: app(k=qk(dtype=pf.PF_F32)))
    refused(bad, lambda: app(k=qk(n_axes=2, pairs=(16, 16, 0))))
    refused(bad, lambda: app(n=4))  # one token a sequence without start
    refused(bad, lambda: app(qo=None))
    refused(bad, lambda: app(x=rows(q=None)))
    for kw in (dict(k=None), dict(v=A + 8), dict(ld_v=120)):
        refused(bad, lambda: app(x=rows(**kw)))
    assert app(n=0, start=A, x=rows(q=0, k=0, v=0)) is None  # no token: nothing to do


def test_workspace_follows_the_split():
    """Two places for each CTA: at most 304, or one for each 64 rows of a key head."""
    size = pf.pf_paged_attn_workspace_size
    assert size(paged(batch=1, max_pages=4)) == 2 * 2 * 2 * 66 * 4
    assert size(paged(batch=64, max_pages=1000)) == size(paged(batch=2048, max_pages=1 << 30)) == 2 * 304 * 2 * 66 * 4


def test_python_refusals():
    """The classes refuse what is not on a GPU, of another type, or no tensor, before the library is called."""
    torch = pytest.importorskip("torch")
    from paper_2608_23463_gb300 import local
    bf, bad = torch.bfloat16, pf.PF_ERR_INVALID_ARG
    q, k = torch.zeros(8, 256, dtype=bf), torch.zeros(8, 128, dtype=bf)
    rope, att = local.QKRope(4, 2, 64), local.WindowAttention(1, 8, 4, 2)
    for x in (q, q.float(), q[:, :128], q[0], None, 7):
        refused(bad, rope.forward, x, k)
        refused(bad, rope.backward, x, k, q, k)
        refused(bad, att.forward, x, k, k)
        refused(bad, att.backward, x, k, k, q, q)
    refused(bad, local.QKRope, 4, 2, 64, torch.zeros(64))
    refused(bad, lambda: local.PagedKVCache(1, 4, 2, 64, 16, 4, 2, device="cpu"))
    with pytest.raises(TypeError):
        local._local.rope_fwd(1, 2)


def test_theta_out_of_range():
    for theta in (1e-301, 1e301, -1.0, float("inf"), float("nan")):
        refused(pf.PF_ERR_INVALID_ARG, pf.pf_qk_rope_fwd, qk(theta=theta), 8, 8, rows(), A, A, None, rows(q=2 * A, k=2 * A))


BASES = dict(q=1 << 28, k=2 << 28, v=3 << 28, out=4 << 28, dout=5 << 28, dq=6 << 28, dk=7 << 28, dv=8 << 28)


def row_bytes(ld, **moved):
    """A matrix's address after another one's: so many rows and bytes on."""
    return {name: BASES[at] + rows * ld * 2 + b for name, (at, rows, b) in moved.items()}


@pytest.mark.parametrize("moved", [
    dict(out=("k", 0, 0)), dict(out=("v", 0, 0)), dict(out=("k", 599, 0)), dict(out=("v", -599, 0)),
    dict(out=("q", 0, 0)), dict(out=("q", 0, 16)), dict(out=("q", 1, 0)), dict(out=("k", 0, 240)), dict(out=("k", -1, 528)),
    dict(q=("out", 0, 256))])
def test_window_forward_overlaps(moved):
    """Results over inputs that are still read, whole or in part."""
    at = {**BASES, **row_bytes(512, **moved)}
    refused(pf.PF_ERR_INVALID_ARG, pf.pf_window_attn_fwd, win(),
            rows(at["q"], at["k"], at["v"], 512, 512, 512), at["out"], 512, A)
    refused(pf.PF_ERR_INVALID_ARG, pf.pf_window_attn_fwd, win(),  # leading dimensions that differ
            rows(at["q"], at["k"], at["v"], 512, 512, 512), at["q"], 520, A)


@pytest.mark.parametrize("moved", [
    dict(dk=("dv", 0, 0)), dict(dq=("dk", 3, 64)), dict(dv=("dq", 0, 496)), dict(dk=("k", 0, 64)), dict(dq=("q", 5, 0)),
    dict(dv=("out", 0, 256)), dict(dq=("dout", -2, -16)), dict(dk=("dv", 599, 0))])
def test_window_backward_overlaps(moved):
    at = {**BASES, **row_bytes(512, **moved)}
    refused(pf.PF_ERR_INVALID_ARG, pf.pf_window_attn_bwd, win(), rows(at["q"], at["k"], at["v"], 512, 512, 512),
            at["out"], 512, A, at["dout"], 512, rows(at["dq"], at["dk"], at["dv"], 512, 512, 512), A, 1 << 40)


@pytest.mark.parametrize("moved", [
    dict(dq=("q", 0, 16)), dict(dq=("k", 0, 0)), dict(dk=("q", 1, 0)), dict(dk=("k", -1, 0)), dict(dq=("dk", 7, 240)),
    dict(dk=("dq", 0, 256))])
def test_rope_overlaps(moved):
    """Each result over its own input or apart from all."""
    at = {**BASES, **row_bytes(512, **moved)}
    z, dz = (rows(at[a], at[b], 0, 512, 512) for a, b in (("q", "k"), ("dq", "dk")))
    far = rows(9 << 28, 10 << 28, 0, 512, 512)
    bad = pf.PF_ERR_INVALID_ARG
    refused(bad, pf.pf_qk_rope_fwd, qk(), 8, 8, z, A, A, None, dz)
    refused(bad, pf.pf_qk_rope_bwd, qk(), 8, 8, z, A, A, None, far, dz, None, None, None, 0)
    refused(bad, pf.pf_qk_rope_bwd, qk(), 8, 8, far, A, A, None, z, dz, None, None, None, 0)
    refused(bad, pf.pf_qk_rope_fwd, qk(), 8, 8, z, A, A, None, rows(at["q"], 11 << 28, 0, 520, 512))


@pytest.mark.parametrize("moved", [dict(out=("q", 0, 16)), dict(out=("k", 0, 0)), dict(out=("v", 2, 240)), dict(out=("q", -1, 0))])
def test_paged_overlaps(moved):
    at = {**BASES, **row_bytes(512, **moved)}
    x, bad = rows(at["q"], at["k"], at["v"], 512, 512, 512), pf.PF_ERR_INVALID_ARG
    refused(bad, pf.pf_paged_append, paged(), qk(), 3, x, A, A, None, None, cache(), at["out"], 512)
    if "q" in {m[0] for m in moved.values()}:
        refused(bad, pf.pf_paged_attn, paged(), at["q"], 512, cache(), at["out"], 512, A, 1 << 30)
    refused(bad, pf.pf_paged_attn, paged(), at["q"], 512, cache(), at["q"], 520, A, 1 << 30)


@pytest.mark.parametrize("x", ["cpu", "shape", None, 7])
def test_refused_backward_keeps_no_workspace(x):
    torch = pytest.importorskip("torch")
    from paper_2608_23463_gb300 import local
    q, k = torch.zeros(8, 256, dtype=torch.bfloat16), torch.zeros(8, 128, dtype=torch.bfloat16)
    x = q if x == "cpu" else q[:, :128] if x == "shape" else x
    att, rope = local.WindowAttention(1, 8, 4, 2), local.QKRope(4, 2, 64)
    rope.w_q = torch.ones(64)  # (a norm's weights on the CPU are refused where the object is made)
    refused(pf.PF_ERR_INVALID_ARG, att.backward, x, k, k, q, q)
    refused(pf.PF_ERR_INVALID_ARG, rope.backward, x, k, q, k)
    assert att.ws is None and rope.ws is None


def test_binding_of_another_torch(monkeypatch):
    """The extension module is compiled again for another torch, and one that is not is refused."""
    torch = pytest.importorskip("torch")
    import importlib

    from paper_2608_23463_gb300 import buildlib, local
    here = buildlib.binding_object()
    assert local._local.built_for == buildlib.binding_tag() and torch.__version__ in here
    monkeypatch.setattr(torch, "__version__", "0.1+other")
    assert buildlib.binding_object() != here
    with pytest.raises(pf.ProxyFormerError) as e:
        importlib.reload(local)
    assert "_local.so" in str(e.value)
    monkeypatch.undo()
    importlib.reload(local)


def test_advance_refuses_other_devices():
    """start on another device than the lengths, or no tensor, before anything is launched."""
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace

    from paper_2608_23463_gb300 import local
    c = local.PagedKVCache.__new__(local.PagedKVCache)
    c.batch, c.len = 2, SimpleNamespace(device=torch.device("cuda", 1))
    other = torch.zeros(3, dtype=torch.int32, device="meta")
    for start in (other, torch.zeros(3, dtype=torch.int32), [0, 1, 2], 7):
        refused(pf.PF_ERR_INVALID_ARG, c.advance, start)
