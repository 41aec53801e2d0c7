"""What the transformer operators refuse, by the host's checks alone: no GPU work."""
import ctypes

import pytest
import torch

from paper_2401_06145_amd import binding as B

P = 4096  # an aligned address that is never read: every call below is refused before any launch


def norm(**kw):
    a = dict(x=P, ld_x=64, res=None, ld_res=0, gamma=P, total=None, ld_sum=0, y=P, ld_y=64, scale=P, ld_scale=1, n=2, c=64,
             dtype=1, bits8=1, eps=1e-6)
    a.update(kw)
    return B.lib().spconv_rms_norm(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), B.SPCONV_EUNSUPPORTED), (dict(n=-1), B.SPCONV_EINVAL), (dict(c=0), B.SPCONV_EINVAL),
    (dict(c=56), B.SPCONV_EUNSUPPORTED), (dict(n=1 << 31), B.SPCONV_EUNSUPPORTED), (dict(eps=-1.0), B.SPCONV_EINVAL),
    (dict(eps=float("nan")), B.SPCONV_EINVAL), (dict(ld_x=63), B.SPCONV_EINVAL), (dict(ld_y=63), B.SPCONV_EINVAL),
    (dict(ld_scale=0), B.SPCONV_EINVAL), (dict(res=P, ld_res=10), B.SPCONV_EINVAL), (dict(total=P, ld_sum=64), B.SPCONV_EINVAL),
    (dict(x=None), B.SPCONV_EINVAL), (dict(gamma=None), B.SPCONV_EINVAL), (dict(y=None), B.SPCONV_EINVAL),
    (dict(scale=None), B.SPCONV_EINVAL), (dict(x=P + 1), B.SPCONV_EINVAL), (dict(scale=P + 2), B.SPCONV_EINVAL),
    (dict(n=0, x=None), B.SPCONV_OK),
])
def test_norm_refusals(kw, status):
    assert norm(**kw) == status
    assert status == B.SPCONV_OK or B.lib().spconv_last_error()


def linear(**kw):
    a = dict(x=P, ld_x=64, xs=P, ld_xs=1, w=P, ld_w=64, ws=P, ld_ws=1, y=P, ld_y=8, m=2, n=8, k=64, dtype=1, relu=0, exact=0)
    a.update(kw)
    return B.lib().spconv_scaled_linear(*a.values(), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=-1), B.SPCONV_EUNSUPPORTED), (dict(m=-1), B.SPCONV_EINVAL), (dict(n=-1), B.SPCONV_EINVAL),
    (dict(k=-16), B.SPCONV_EINVAL), (dict(k=40), B.SPCONV_EUNSUPPORTED), (dict(ld_x=72), B.SPCONV_EUNSUPPORTED),
    (dict(ld_w=72), B.SPCONV_EUNSUPPORTED), (dict(ld_x=48), B.SPCONV_EINVAL), (dict(ld_w=48), B.SPCONV_EINVAL),
    (dict(ld_y=7), B.SPCONV_EINVAL), (dict(ld_xs=0), B.SPCONV_EINVAL), (dict(ld_ws=0), B.SPCONV_EINVAL),
    (dict(m=1 << 31), B.SPCONV_EUNSUPPORTED), (dict(x=None), B.SPCONV_EINVAL), (dict(xs=None), B.SPCONV_EINVAL),
    (dict(w=None), B.SPCONV_EINVAL), (dict(ws=None), B.SPCONV_EINVAL), (dict(y=None), B.SPCONV_EINVAL),
    (dict(x=P + 8), B.SPCONV_EINVAL), (dict(w=P + 8), B.SPCONV_EINVAL), (dict(y=P + 1), B.SPCONV_EINVAL),
    (dict(xs=P + 1), B.SPCONV_EINVAL), (dict(ld_x=(1 << 23) + 16), B.SPCONV_EUNSUPPORTED),
    (dict(ld_w=(1 << 23) + 16), B.SPCONV_EUNSUPPORTED), (dict(ld_xs=(1 << 21) + 1), B.SPCONV_EUNSUPPORTED), (dict(m=0, x=None), B.SPCONV_OK), (dict(n=0, w=None, ld_y=0), B.SPCONV_OK),
])
def test_linear_refusals(kw, status):
    assert linear(**kw) == status
    assert status == B.SPCONV_OK or B.lib().spconv_last_error()


def attention_args(**kw):
    a = dict(d_q=P, d_k=P, d_v=P, d_out=P, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, out_row=256,
             out_head=64, d_q_start=P, d_k_start=P, d_k_len=None, d_prefix=None, d_slopes=None, d_q_pos=None, d_k_pos=None,
             n_q=2, n_k=9, n_docs=1, max_q=2, max_k=9, heads=4, kv_heads=2, head_dim=64, dtype=1, causal=1, scale=0.125,
             cap=0.0)
    a.update(kw)
    return B.AttentionArgs(**a)


BAD = [
    (dict(dtype=4), B.SPCONV_EUNSUPPORTED), (dict(n_q=-1), B.SPCONV_EINVAL), (dict(n_k=-1), B.SPCONV_EINVAL),
    (dict(n_docs=-1), B.SPCONV_EINVAL), (dict(max_k=-1), B.SPCONV_EINVAL), (dict(kv_heads=3), B.SPCONV_EINVAL),
    (dict(kv_heads=0), B.SPCONV_EINVAL), (dict(heads=0), B.SPCONV_EINVAL), (dict(head_dim=4), B.SPCONV_EUNSUPPORTED),
    (dict(head_dim=60), B.SPCONV_EUNSUPPORTED), (dict(head_dim=264), B.SPCONV_EUNSUPPORTED), (dict(scale=0.0), B.SPCONV_EINVAL),
    (dict(scale=float("inf")), B.SPCONV_EINVAL), (dict(scale=float("nan")), B.SPCONV_EINVAL), (dict(cap=-1.0), B.SPCONV_EINVAL),
    (dict(cap=float("nan")), B.SPCONV_EINVAL), (dict(d_q_pos=P), B.SPCONV_EINVAL), (dict(d_q_pos=P, d_k_pos=P), B.SPCONV_EINVAL),
    (dict(n_q=1 << 31), B.SPCONV_EUNSUPPORTED), (dict(n_k=1 << 31), B.SPCONV_EUNSUPPORTED),
    (dict(heads=65536, kv_heads=65536), B.SPCONV_EUNSUPPORTED), (dict(max_k=(1 << 30) + 1), B.SPCONV_EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(d_q=None), B.SPCONV_EINVAL), (dict(d_k=None), B.SPCONV_EINVAL), (dict(d_v=None), B.SPCONV_EINVAL),
    (dict(d_out=None), B.SPCONV_EINVAL), (dict(d_q_start=None), B.SPCONV_EINVAL), (dict(d_k_start=None), B.SPCONV_EINVAL),
    (dict(d_q=P + 8), B.SPCONV_EINVAL), (dict(d_out=P + 8), B.SPCONV_EINVAL), (dict(q_row=252), B.SPCONV_EUNSUPPORTED),
    (dict(k_row=-128), B.SPCONV_EUNSUPPORTED), (dict(out_head=56), B.SPCONV_EINVAL), (dict(out_row=32), B.SPCONV_EINVAL),
    (dict(k_row=(1 << 24) + 8), B.SPCONV_EUNSUPPORTED), (dict(v_row=(1 << 24) + 8), B.SPCONV_EUNSUPPORTED),
    (dict(max_q=0), B.SPCONV_EINVAL), (dict(n_q=0, d_q=None), B.SPCONV_OK), (dict(n_docs=0), B.SPCONV_OK),
])
def test_attention_refusals(kw, status):
    assert B.lib().spconv_attention(ctypes.byref(attention_args(**kw)), None, 0, None) == status
    assert status == B.SPCONV_OK or B.lib().spconv_last_error()


@pytest.mark.parametrize("kw", [k for k, _ in BAD])
def test_no_workspace_for_what_is_refused(kw):
    assert B.spconv_attention_workspace_bytes(attention_args(**kw)) == 0


def test_attention_workspace():
    assert B.lib().spconv_attention(None, None, 0, None) == B.SPCONV_EINVAL
    assert B.lib().spconv_attention_workspace_bytes(None) == 0
    assert B.spconv_attention_workspace_bytes(attention_args()) == 0  # nine keys: not split
    long = attention_args(n_q=1, max_q=1, n_k=20_000, max_k=20_000)
    need = B.spconv_attention_workspace_bytes(long)
    assert need >= 2 * 4 * (64 + 2) * 4  # two parts of four heads at least
    run = B.lib().spconv_attention
    assert run(ctypes.byref(long), None, 0, None) == B.SPCONV_ENOSPC
    assert run(ctypes.byref(long), P, need - 1, None) == B.SPCONV_ENOSPC
    assert run(ctypes.byref(long), P + 16, need, None) == B.SPCONV_EINVAL


def test_binding_refuses_other_shapes():
    x = torch.zeros((4, 32), dtype=torch.float16)
    gamma = torch.ones(32, dtype=torch.float16)
    for bad in (dict(gamma=gamma[:16]), dict(gamma=gamma.float()), dict(residual=x[:2]), dict(residual=x.float()),
                dict(x=x.t()), dict(x=x.double(), gamma=gamma.double())):
        with pytest.raises(ValueError):
            B.rms_norm(**{"x": x, "gamma": gamma, **bad})
    q8 = torch.zeros((4, 32), dtype=torch.uint8).view(B.E4M3)
    s = torch.ones((4, 1))
    for bad in (dict(x=x), dict(w=q8[:, :16]), dict(x_scale=s[:2]), dict(w_scale=s), dict(x_scale=s.double()),
                dict(dtype=torch.float64)):
        with pytest.raises(ValueError):
            B.scaled_linear(**{"x": q8, "x_scale": s, "w": q8, "w_scale": s[:1], "dtype": torch.float16, **bad})
    q = torch.zeros((4, 2, 32), dtype=torch.float16)
    at = torch.tensor([0, 4], dtype=torch.int32)
    for bad in (dict(k=q.float()), dict(v=q[:2]), dict(k=q[..., :16], v=q[..., :16]), dict(q=q.transpose(1, 2)),
                dict(q_start=at.long()), dict(k_len=at), dict(prefix=at), dict(slopes=torch.ones(3)),
                dict(slopes=torch.ones(2, dtype=torch.float64)), dict(q_pos=torch.zeros((4, 3), dtype=torch.int32)),
                dict(q=q.double())):
        with pytest.raises(ValueError):
            B.attention(**{"q": q, "k": q, "v": q, "q_start": at, "k_start": at, "max_q": 4, "max_k": 4, **bad})


@pytest.mark.parametrize("kw", [
    dict(m=(1 << 31) - 1, n=1, k=16), dict(m=(1 << 31) - 1, n=1, k=16, exact=1), dict(m=(1 << 31) - 1, n=1, k=16, dtype=0),
    dict(m=1, n=(1 << 31) - 1, k=16), dict(m=40, n=(1 << 31) - 1, k=2048, ld_x=2048, ld_w=2048, ld_xs=16, ld_ws=16),
    dict(m=(1 << 31) - 1, n=(1 << 31) - 1, k=16),
])
def test_product_of_more_than_one_launch_takes(kw):
    """2^32 threads and more would start as fewer, without an error."""
    assert linear(**{"ld_y": 1 << 31, **kw}) == B.SPCONV_EUNSUPPORTED
    assert b"launch" in B.lib().spconv_last_error()


@pytest.mark.parametrize("kw", [
    dict(n_q=(1 << 31) - 1, max_q=1 << 20, heads=128, kv_heads=2, q_row=8192, out_row=8192),
    dict(n_q=70, n_docs=(1 << 31) - 1, max_q=40), dict(n_q=1 << 24, n_docs=1 << 24, max_q=40, heads=1, kv_heads=1, max_k=9),
    dict(n_q=70, n_docs=1 << 28, max_q=1, heads=65535, kv_heads=65535, q_row=65535 * 64, out_row=65535 * 64),
])
def test_attention_of_more_than_one_launch_takes(kw):
    assert B.lib().spconv_attention(ctypes.byref(attention_args(**kw)), P, 1 << 62, None) == B.SPCONV_EUNSUPPORTED
    assert b"launch" in B.lib().spconv_last_error()


def test_binding_refuses_what_needs_gradients():
    """Forward only: a call that autograd would have to record is refused, and is taken without it."""
    x = torch.zeros((4, 32), dtype=torch.float16)
    q = torch.zeros((4, 2, 32), dtype=torch.float16)
    at, slopes = torch.tensor([0, 4], dtype=torch.int32), torch.ones(2)
    q8, s = torch.zeros((4, 32), dtype=torch.uint8).view(B.E4M3), torch.ones((4, 1))
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    norm = lambda **kw: B.rms_norm(**{"x": x, "gamma": x[0], **kw})  # noqa: E731
    linear = lambda **kw: B.scaled_linear(**{"x": q8, "x_scale": s, "w": q8, "w_scale": s[:1], "dtype": torch.float16, **kw})  # noqa: E731
    attend = lambda **kw: B.attention(**{"q": q, "k": q, "v": q, "q_start": at, "k_start": at, "max_q": 4, "max_k": 4,  # noqa: E731
                                         "slopes": slopes, **kw})
    for call, kw in ((norm, dict(x=leaf(x))), (norm, dict(gamma=leaf(x[0]))), (norm, dict(residual=leaf(x) * 2)),
                     (linear, dict(x_scale=leaf(s))), (linear, dict(w_scale=leaf(s[:1]))), (attend, dict(q=leaf(q))),
                     (attend, dict(k=leaf(q))), (attend, dict(v=leaf(q))), (attend, dict(slopes=leaf(slopes)))):
        with pytest.raises(ValueError, match="gradient"):
            call(**kw)
        with torch.no_grad(), pytest.raises(ValueError, match="GPU|device"):  # taken, as far as this test's CPU tensors go
            call(**kw)
    import torch.autograd.forward_ad as fwd

    with fwd.dual_level():
        with pytest.raises(ValueError, match="gradient"):
            norm(x=fwd.make_dual(x, torch.ones_like(x)))


def test_binding_refuses_rows_of_more_than_31_bits():
    """Their number of columns must not wrap to a small one."""
    x = torch.empty((1, (1 << 32) + 16), dtype=torch.float16)  # never touched
    with pytest.raises(ValueError, match="columns"):
        B.rms_norm(x, x[0])


@pytest.mark.parametrize("exact", [False, True])
def test_transformer_asks_for_exact_products(exact, monkeypatch):
    from paper_2401_06145_amd import transformer

    asked = []
    monkeypatch.setattr(B, "scaled_linear", lambda *a, **kw: asked.append(kw["exact"]))
    model = transformer.Transformer(transformer.Config(width=32, heads=2, kv_heads=1, layers=1, inner=32, exact=exact), device="cpu")
    model._linear((None, None), model.layers[0]["qkv"])
    assert asked == [exact]
