"""What the operators of a paged cache refuse, by the host's checks alone: no GPU work."""
import ctypes

import pytest
import torch

from paper_2401_06145_amd import binding as B
from tests.test_transformer_abi import BAD, attention_args

P = 4096  # an aligned address that is never read: every call below is refused before any launch


def rotation(**kw):
    a = dict(d_q=P, d_q_out=P, d_k=P, d_k_out=P, q_row=256, q_head=64, q_out_row=256, q_out_head=64, k_row=128, k_head=64,
             k_out_row=128, k_out_head=64, d_q_gamma=P, d_k_gamma=None, d_pos=P, d_freq=P, n=2, heads=4, kv_heads=2,
             head_dim=64, rotated=64, dtype=1, interleaved=0, voxels=0, eps=1e-6, gain=1.0)
    a.update(kw)
    return B.lib().spconv_rotate_heads(ctypes.byref(B.Rotation(**a)), None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), B.SPCONV_EUNSUPPORTED), (dict(n=-1), B.SPCONV_EINVAL), (dict(heads=0), B.SPCONV_EINVAL),
    (dict(kv_heads=-1), B.SPCONV_EINVAL), (dict(n=1 << 31), B.SPCONV_EUNSUPPORTED), (dict(heads=65536), B.SPCONV_EUNSUPPORTED),
    (dict(kv_heads=65536), B.SPCONV_EUNSUPPORTED), (dict(head_dim=0), B.SPCONV_EUNSUPPORTED),
    (dict(head_dim=257, rotated=64), B.SPCONV_EUNSUPPORTED), (dict(rotated=63), B.SPCONV_EINVAL), (dict(rotated=66), B.SPCONV_EINVAL),
    (dict(rotated=-2), B.SPCONV_EINVAL), (dict(eps=-1.0), B.SPCONV_EINVAL), (dict(eps=float("nan")), B.SPCONV_EINVAL),
    (dict(gain=float("inf")), B.SPCONV_EINVAL), (dict(d_q=None), B.SPCONV_EINVAL), (dict(d_q_out=None), B.SPCONV_EINVAL),
    (dict(d_k=None), B.SPCONV_EINVAL), (dict(d_k_out=None), B.SPCONV_EINVAL), (dict(d_pos=None), B.SPCONV_EINVAL),
    (dict(d_freq=None), B.SPCONV_EINVAL), (dict(d_q=P + 1), B.SPCONV_EINVAL), (dict(d_k_out=P + 1), B.SPCONV_EINVAL),
    (dict(d_q_gamma=P + 1), B.SPCONV_EINVAL), (dict(d_pos=P + 2), B.SPCONV_EINVAL), (dict(d_freq=P + 4), B.SPCONV_EINVAL),
    (dict(q_row=-256), B.SPCONV_EINVAL), (dict(k_head=-64), B.SPCONV_EINVAL), (dict(q_out_row=63), B.SPCONV_EINVAL),
    (dict(k_out_head=63), B.SPCONV_EINVAL), (dict(n=0, d_q=None), B.SPCONV_OK),
])
def test_rotation_refusals(kw, status):
    assert rotation(**kw) == status
    assert status == B.SPCONV_OK or B.lib().spconv_last_error()


def pages(**kw):
    a = dict(d_k=P, d_v=P, d_k_scale=None, d_v_scale=None, d_table=P, n_pages=9, n_docs=1, table_row=4, page=16, kv_heads=2,
             head_dim=64)
    a.update(kw)
    return B.PagesArgs(**a)


def write(p=None, **kw):
    a = dict(k=P, k_row=128, k_head=64, v=P, v_row=128, v_head=64, start=P, len=P, n=3, dtype=1)
    a.update(kw)
    return B.lib().spconv_cache_write(None if p is None else ctypes.byref(p), *a.values(), None)


def read(p=None, **kw):
    a = dict(k=P, k_row=128, k_head=64, v=P, v_row=128, v_head=64, start=P, n=3, dtype=1)
    a.update(kw)
    return B.lib().spconv_cache_read(None if p is None else ctypes.byref(p), *a.values(), None)


def attend(p=None, **kw):
    return B.lib().spconv_cached_attention(None if p is None else ctypes.byref(p), ctypes.byref(attention_args(d_k_len=P, **kw)),
                                           None, 0, None)


BAD_PAGES = [
    (dict(n_pages=-1), B.SPCONV_EINVAL), (dict(n_docs=-1), B.SPCONV_EINVAL), (dict(table_row=-1), B.SPCONV_EINVAL),
    (dict(n_pages=1 << 31), B.SPCONV_EUNSUPPORTED), (dict(kv_heads=0), B.SPCONV_EINVAL), (dict(kv_heads=65536), B.SPCONV_EUNSUPPORTED),
    (dict(head_dim=4), B.SPCONV_EUNSUPPORTED), (dict(head_dim=60), B.SPCONV_EUNSUPPORTED), (dict(head_dim=264), B.SPCONV_EUNSUPPORTED),
    (dict(d_k_scale=P, d_v_scale=P, head_dim=72), B.SPCONV_EUNSUPPORTED), (dict(d_k_scale=P), B.SPCONV_EINVAL),
    (dict(d_v_scale=P), B.SPCONV_EINVAL), (dict(page=0), B.SPCONV_EUNSUPPORTED), (dict(page=-16), B.SPCONV_EUNSUPPORTED),
    (dict(page=48), B.SPCONV_EUNSUPPORTED), (dict(page=1 << 17), B.SPCONV_EUNSUPPORTED),
    (dict(table_row=(1 << 26) + 1), B.SPCONV_EUNSUPPORTED), (dict(d_k=None), B.SPCONV_EINVAL), (dict(d_v=None), B.SPCONV_EINVAL),
    (dict(d_table=None), B.SPCONV_EINVAL), (dict(d_k=P + 8), B.SPCONV_EINVAL), (dict(d_v=P + 8), B.SPCONV_EINVAL),
    (dict(d_table=P + 2), B.SPCONV_EINVAL), (dict(d_k_scale=P + 2, d_v_scale=P), B.SPCONV_EINVAL),
]


@pytest.mark.parametrize("call", [write, read])
@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_page_refusals(kw, status, call):
    assert call(pages(**kw)) == status
    assert B.lib().spconv_last_error()


@pytest.mark.parametrize("kw,status", BAD_PAGES)
def test_page_refusals_of_attention(kw, status):
    same = {k: kw[k] for k in ("kv_heads", "head_dim", "n_docs") if k in kw}
    if "kv_heads" in same:
        same["heads"] = max(1, same["kv_heads"])
    assert attend(pages(**kw), **same) == status
    assert B.lib().spconv_last_error()


@pytest.mark.parametrize("call", [write, read])
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), B.SPCONV_EUNSUPPORTED), (dict(n=-1), B.SPCONV_EINVAL), (dict(n=1 << 31), B.SPCONV_EUNSUPPORTED),
    (dict(k=None), B.SPCONV_EINVAL), (dict(v=None), B.SPCONV_EINVAL), (dict(start=None), B.SPCONV_EINVAL),
    (dict(k=P + 8), B.SPCONV_EINVAL), (dict(v=P + 2), B.SPCONV_EINVAL), (dict(k_row=124), B.SPCONV_EUNSUPPORTED),
    (dict(v_head=-64), B.SPCONV_EUNSUPPORTED), (dict(n=0, k=None), B.SPCONV_OK),
])
def test_row_refusals(kw, status, call):
    assert call(None) == B.SPCONV_EINVAL
    assert call(pages(), **kw) == status


def test_write_and_read_refusals_of_their_own():
    assert write(pages(), len=None) == B.SPCONV_EINVAL
    assert read(pages(), k_row=56) == B.SPCONV_EINVAL and read(pages(), v_head=56) == B.SPCONV_EINVAL
    assert write(pages(n_docs=0)) == B.SPCONV_OK and read(pages(n_docs=0, d_table=None)) == B.SPCONV_OK


@pytest.mark.parametrize("kw,status", BAD + [
    (dict(d_q=None), B.SPCONV_EINVAL), (dict(d_out=None), B.SPCONV_EINVAL), (dict(d_q_start=None), B.SPCONV_EINVAL),
    (dict(d_q=P + 8), B.SPCONV_EINVAL), (dict(d_out=P + 8), B.SPCONV_EINVAL), (dict(q_row=252), B.SPCONV_EUNSUPPORTED),
    (dict(out_head=56), B.SPCONV_EINVAL), (dict(out_row=32), B.SPCONV_EINVAL), (dict(max_q=0), B.SPCONV_EINVAL),
    (dict(n_docs=2), B.SPCONV_EINVAL), (dict(head_dim=32), B.SPCONV_EINVAL), (dict(kv_heads=4), B.SPCONV_EINVAL),
    (dict(d_q_pos=P, d_k_pos=P, d_slopes=P), B.SPCONV_EUNSUPPORTED), (dict(n_q=0, d_q=None), B.SPCONV_OK),
    (dict(d_k=None, d_v=None, d_k_start=None, d_q=None), B.SPCONV_EINVAL),
])
def test_cached_attention_refusals(kw, status):
    assert attend(pages(), **kw) == status
    assert B.spconv_cached_attention_workspace_bytes(pages(), attention_args(d_k_len=P, **kw)) == 0


def test_cached_attention_workspace():
    assert B.lib().spconv_cached_attention(None, ctypes.byref(attention_args()), None, 0, None) == B.SPCONV_EINVAL
    assert B.lib().spconv_cached_attention(ctypes.byref(pages()), None, None, 0, None) == B.SPCONV_EINVAL
    p, long = pages(table_row=2000), attention_args(n_q=1, max_q=1, max_k=20_000, d_k_len=P)
    need = B.spconv_cached_attention_workspace_bytes(p, long)
    assert need >= 2 * 4 * (64 + 2) * 4  # two parts of four heads at least
    run = B.lib().spconv_cached_attention
    assert run(ctypes.byref(p), ctypes.byref(long), None, 0, None) == B.SPCONV_ENOSPC
    assert run(ctypes.byref(p), ctypes.byref(long), P, need - 1, None) == B.SPCONV_ENOSPC
    assert run(ctypes.byref(p), ctypes.byref(long), P + 16, need, None) == B.SPCONV_EINVAL
    long.d_k_len = None
    assert run(ctypes.byref(p), ctypes.byref(long), P, need, None) == B.SPCONV_EINVAL


F16 = torch.float16


def cache_of(dtype=F16, bits8=False):
    return B.Pages.make(4, 8, 2, 32, dtype, bits8, "cpu")


def test_binding_refuses_other_shapes():
    q, k = torch.zeros((4, 4, 32), dtype=F16), torch.zeros((4, 2, 32), dtype=F16)
    at, lens, table = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([4], dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32)
    pos, freq, gamma = torch.arange(4, dtype=torch.int32), torch.ones(16, dtype=torch.float64), torch.ones(32, dtype=F16)
    rotate = lambda **kw: B.rotate_heads(**{"q": q, "k": k, "pos": pos, "freq": freq, **kw})  # noqa: E731
    write = lambda **kw: B.cache_write(**{"cache": cache_of(), "k": k, "v": k, "q_start": at, "k_len": lens, "table": table, **kw})  # noqa: E731
    read = lambda **kw: B.cache_read(**{"cache": cache_of(), "start": at, "table": table, "rows": 4, "dtype": F16, **kw})  # noqa: E731
    attend = lambda **kw: B.cached_attention(**{"q": q, "cache": cache_of(), "q_start": at, "k_len": lens, "table": table,  # noqa: E731
                                                "max_q": 4, "max_k": 4, **kw})
    c, c8 = cache_of(), cache_of(bits8=True)
    assert c8.page == 8 and c8.k.dtype == B.E4M3 and c.k_scale is None
    pages = [dict(cache=B.Pages(c.k, c.v[:3])), dict(cache=B.Pages(c.k, c.v.float())), dict(cache=B.Pages(c8.k, c8.v)),
             dict(cache=B.Pages(c.k, c.v, c8.k_scale, c8.v_scale)), dict(cache=B.Pages(c8.k, c8.v, c8.k_scale[:3], c8.v_scale)),
             dict(cache=B.Pages(c8.k, c8.v, c8.k_scale.double(), c8.v_scale)), dict(cache=B.Pages(c.k[0], c.v[0])),
             dict(cache=B.Pages(c.k.transpose(2, 3), c.v.transpose(2, 3))), dict(cache=cache_of(torch.float32)),
             dict(table=table[0]), dict(table=table.long()), dict(table=torch.zeros((2, 2), dtype=torch.int32))]
    for call, bads in (
            (rotate, [dict(k=k[:3]), dict(k=k.float()), dict(k=k[..., :16]), dict(q=q[0]), dict(q=q.transpose(1, 2)), dict(q=q.double()),
                      dict(pos=pos.long()), dict(pos=pos[:3]), dict(pos=torch.zeros((4, 3), dtype=torch.int32)), dict(freq=freq.float()),
                      dict(freq=freq[None]), dict(q_gamma=gamma[:8]), dict(k_gamma=gamma.float()), dict(q_gamma=torch.ones((2, 32), dtype=F16))]),
            (write, pages + [dict(k=k[:, :1], v=k[:, :1]), dict(v=k[:3]), dict(v=k.float()), dict(k=k[..., :16], v=k[..., :16]),
                             dict(q_start=lens), dict(k_len=at), dict(q_start=at.long()), dict(k=k.transpose(1, 2))]),
            (read, pages + [dict(start=lens), dict(start=at.long()), dict(rows=-1), dict(dtype=torch.float64), dict(dtype=torch.float32),
                            dict(rows=1 << 31)]),
            (attend, pages + [dict(q=q[..., :16]), dict(q=q.float()), dict(q=q[0]), dict(q_start=lens), dict(k_len=at), dict(prefix=at),
                              dict(slopes=torch.ones(3)), dict(max_q=1 << 31)])):
        with pytest.raises(ValueError, match="GPU|device"):  # taken, as far as this test's CPU tensors go
            call()
        for bad in bads:
            with pytest.raises((ValueError, TypeError)) as e:
                call(**bad)
            assert "GPU" not in str(e.value), bad
    for call in (write, attend):
        for none in ("q_start", "k_len"):
            with pytest.raises(ValueError, match="tensor"):
                call(**{none: None})


def test_binding_refuses_what_needs_gradients():
    q, k = torch.zeros((4, 4, 32), dtype=F16), torch.zeros((4, 2, 32), dtype=F16)
    at, lens, table = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([4], dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32)
    pos, freq, gamma = torch.arange(4, dtype=torch.int32), torch.ones(16, dtype=torch.float64), torch.ones(32, dtype=F16)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    c = cache_of()
    grown = B.Pages(leaf(c.k), c.v)
    for call in (lambda: B.rotate_heads(leaf(q), k, pos, freq), lambda: B.rotate_heads(q, leaf(k), pos, freq),
                 lambda: B.rotate_heads(q, k, pos, leaf(freq)), lambda: B.rotate_heads(q, k, pos, freq, leaf(gamma)),
                 lambda: B.rotate_heads(q, k, pos, freq, None, leaf(gamma)), lambda: B.cache_write(c, leaf(k), k, at, lens, table),
                 lambda: B.cache_write(c, k, leaf(k), at, lens, table), lambda: B.cache_write(grown, k, k, at, lens, table),
                 lambda: B.cache_read(grown, at, table, 4, F16), lambda: B.cached_attention(leaf(q), c, at, lens, table, 4, 4),
                 lambda: B.cached_attention(q, grown, at, lens, table, 4, 4),
                 lambda: B.cached_attention(q, c, at, lens, table, 4, 4, slopes=leaf(torch.ones(4)))):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU|device"):
            call()


@pytest.mark.parametrize("call", [
    lambda: rotation(n=(1 << 31) - 1), lambda: rotation(n=(1 << 31) - 1, heads=65535, kv_heads=0),
    lambda: write(pages(), n=(1 << 31) - 1), lambda: read(pages(kv_heads=64), n=(1 << 31) - 1, k_row=4096, v_row=4096),
    lambda: attend(pages(n_docs=1 << 24), n_q=1 << 24, n_docs=1 << 24, max_q=40, heads=2, max_k=9),
    lambda: attend(pages(n_docs=1 << 26), n_q=70, n_docs=1 << 26, max_q=40, max_k=9),
])
def test_more_than_one_launch_takes(call):
    """2^32 threads and more would start as fewer, without an error."""
    assert call() == B.SPCONV_EUNSUPPORTED
    assert b"launch" in B.lib().spconv_last_error()


def test_queries_of_a_key_head_have_31_bits():
    assert attend(pages(kv_heads=1), n_q=1 << 30, kv_heads=1, max_q=1 << 30) == B.SPCONV_EUNSUPPORTED
    assert B.spconv_cached_attention_workspace_bytes(pages(kv_heads=1), attention_args(n_q=1 << 30, kv_heads=1, max_q=1 << 30)) == 0
    assert write(pages(kv_heads=1 << 12, page=1 << 16, head_dim=64, table_row=1)) == B.SPCONV_EUNSUPPORTED


def test_rows_of_packed_keys_are_no_part_of_cached_attention():
    """n_k may be any number that the packed call takes; nothing goes by it."""
    p = pages(table_row=2000)
    need = [B.spconv_cached_attention_workspace_bytes(p, attention_args(n_q=1, max_q=1, max_k=20_000, d_k_len=P, n_k=n, d_k=None,
                                                                        d_v=None, d_k_start=None, k_row=3, v_head=-1))
            for n in (0, 9, 20_000, (1 << 31) - 1)]
    assert need[0] > 0 and len(set(need)) == 1
