"""What the served decoding step's entry points refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from paper_2505_19342_amd import binding as B

GOOD = dict(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=32, n_pages=40, n_seqs=4, max_pages=8, n_tokens=5)
A = 1 << 20                       # an address: 16-byte aligned, never read here


def cache(**change):
    raw = {k: change.pop(k) for k in list(change) if k in ("dtype_raw",)}
    d = B.cache_desc(**{**GOOD, **change})
    if raw:
        d.dtype = raw["dtype_raw"]
    return d


def append(desc, q=A, k=A, q_out=A, pages=A, table=A):
    return B.load().astra_cache_append(ctypes.byref(desc), table, A, A, None, q, k, A, q_out, pages, A, A, A, None)


def attend(desc, q=A, prior=None, prior_lse=None, out=A, ws=A, ws_bytes=1 << 40, first=A):
    return B.load().astra_cache_attention(ctypes.byref(desc), A, A, first, q, A, A, A, A, prior, prior_lse, out, None, ws, ws_bytes, None)


NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5


@pytest.mark.parametrize("change, rc", [
    (dict(dtype_raw=2), DTYPE), (dict(n_kv_heads=3), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_q_heads=-8), SHAPE), (dict(head_dim=96), UNSUPPORTED),
    (dict(head_dim=0), SHAPE), (dict(page_size=48), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=256), UNSUPPORTED), (dict(page_size=-16), SHAPE),
    (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(table_stride=7), SHAPE),
    (dict(n_seqs=1025), UNSUPPORTED), (dict(max_pages=1 << 26), SHAPE), (dict(rope_base=-1.0), SHAPE), (dict(rope_base=float("nan")), SHAPE),
    (dict(rope_base=float("inf")), SHAPE), (dict(scale=-0.1), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(q_stride=1020), SHAPE), (dict(q_stride=1028), UNSUPPORTED), (dict(k_stride=255), SHAPE), (dict(v_stride=260), UNSUPPORTED),
    (dict(q_stride=-1024), SHAPE),
])
def test_descriptors_of_the_cache(change, rc):
    assert append(cache(**change)) == rc and attend(cache(**change)) == rc
    assert B.astra_cache_attention_workspace_bytes(cache(**change)) == 0
    assert B.astra_cache_attention_workspace_bytes(cache()) > 0


def test_addresses_of_the_cache():
    lib, d = B.load(), cache()
    assert lib.astra_cache_append(None, *[None] * 14) == NULL and lib.astra_cache_attention(None, *[None] * 13, 0, None) == NULL
    assert append(d, k=None) == NULL and append(d, q=None) == NULL and append(d, q_out=None) == NULL and append(d, table=None) == NULL
    assert append(d, k=A + 8) == UNSUPPORTED and append(d, pages=A + 4) == UNSUPPORTED and append(d, q_out=A + 2) == UNSUPPORTED
    assert attend(d, q=None) == NULL and attend(d, first=None) == NULL and attend(d, prior=A) == NULL and attend(d, prior_lse=A) == NULL and attend(d, out=None) == NULL
    assert attend(d, out=A + 8) == UNSUPPORTED and attend(d, q=A + 4) == UNSUPPORTED
    assert attend(d, ws=None) == WORKSPACE and attend(d, ws_bytes=B.astra_cache_attention_workspace_bytes(d) - 1) == WORKSPACE
    # nothing to do: nothing is asked for
    for nothing in (cache(n_tokens=0), cache(n_seqs=0)):
        assert lib.astra_cache_append(ctypes.byref(nothing), *[None] * 13) == 0
        assert lib.astra_cache_attention(ctypes.byref(nothing), *[None] * 13, 0, None) == 0


def w4(desc, x=A, n=3, codes=A, scales=A, y=A):
    return B.load().astra_w4_linear(ctypes.byref(desc), x, n, codes, scales, None, None, y, None)


def test_products_with_four_bits():
    good = ("bf16", 512, 100, 64)
    assert B.load().astra_w4_linear(None, *[None] * 1, 1, *[None] * 6) == NULL
    for args, rc in ((("bf16", 500, 100, 64), SHAPE), (("bf16", 512, 0, 64), SHAPE), (("bf16", 0, 100, 64), SHAPE), (("bf16", 512, 100, 16), UNSUPPORTED),
                     (("bf16", 512, 100, 256), UNSUPPORTED), (("bf16", 512, 100, 0), SHAPE), (("bf16", 1 << 25, 100, 64), UNSUPPORTED)):
        assert w4(B.w4_desc(*args)) == rc, args
    assert w4(B.w4_desc(*good, x_stride=500)) == SHAPE and w4(B.w4_desc(*good, x_stride=516)) == UNSUPPORTED
    d = B.w4_desc(*good)
    d.y_dtype = 7
    assert w4(d) == DTYPE
    d = B.w4_desc(*good)
    assert w4(d, n=-1) == SHAPE and w4(d, n=(1 << 20) + 1) == SHAPE and w4(d, n=0) == 0
    assert w4(d, x=None) == NULL and w4(d, codes=None) == NULL and w4(d, scales=None) == NULL and w4(d, y=None) == NULL
    assert w4(d, x=A + 8) == UNSUPPORTED and w4(d, codes=A + 1) == UNSUPPORTED


class Tensor:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype, device=0, stride=None):
        import torch
        self.meta = torch.empty_strided(shape, stride, dtype=dtype, device="meta") if stride else torch.empty(shape, dtype=dtype, device="meta")
        self.is_cuda, self.device = True, device
        self.dtype, self.shape = dtype, self.meta.shape

    def get_device(self):
        return self.device

    def __getattr__(self, name):
        return getattr(self.meta, name)

    def __getitem__(self, i):
        return self.meta[i]

    def data_ptr(self):
        return A


def test_tensors_that_do_not_fit(monkeypatch):
    import torch
    bf, i32, f32, u8 = torch.bfloat16, torch.int32, torch.float32, torch.uint8
    monkeypatch.setattr(B, "_types", None)
    monkeypatch.setattr(B, "_types", B._dtypes()[:4] + (lambda: 0, lambda device: None))
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0 if name != "astra_status_string" else b"?"
    monkeypatch.setattr(B, "load", lambda build_if_missing=True: Library())
    d = cache(k_stride=512)
    good = dict(page_table=Tensor((4, 8), i32), lens=Tensor((4,), i32), first_row=Tensor((5,), i32), pos_shift=None, q=Tensor((5, 8, 128), bf),
                k=Tensor((5, 256), bf, stride=(512, 1)), v=Tensor((5, 2, 128), bf), q_out=Tensor((5, 8, 128), bf), k_pages=Tensor((40, 2, 32, 128), u8),
                v_pages=Tensor((40, 2, 32, 128), torch.float8_e4m3fn), k_scales=Tensor((40, 2), f32), v_scales=Tensor((40, 2), f32))
    B.astra_cache_append(d, **good)
    assert called == ["astra_cache_append"]
    for change in (dict(page_table=Tensor((4, 7), i32)), dict(lens=Tensor((4,), torch.int64)), dict(first_row=Tensor((4,), i32)), dict(q=Tensor((5, 8, 128), f32)),
                   dict(q=Tensor((4, 8, 128), bf)), dict(k=Tensor((5, 256), bf)), dict(k=Tensor((5, 256), bf, stride=(500, 1))), dict(k=Tensor((5, 256), bf, stride=(512, 2))),
                   dict(v=Tensor((5, 256), bf, stride=(512, 1))), dict(k_pages=Tensor((39, 2, 32, 128), u8)), dict(k_scales=Tensor((40,), f32)),
                   dict(v_scales=Tensor((40, 2), bf)), dict(q=Tensor((5, 8, 128), bf, device=1)), dict(pos_shift=Tensor((3,), i32))):
        with pytest.raises(B.AstraError):
            B.astra_cache_append(d, **{**good, **change})
    assert called == ["astra_cache_append"]
    w = B.w4_desc("bf16", 512, 100, 64, "f32")
    fit = dict(x=Tensor((3, 512), bf), n_tokens=3, codes=Tensor((100, 256), u8), scales=Tensor((100, 8), bf), zeros=None, bias=None, y=Tensor((3, 100), f32))
    B.astra_w4_linear(w, **fit)
    for change in (dict(n_tokens=4), dict(codes=Tensor((100, 255), u8)), dict(scales=Tensor((100, 8), f32)), dict(zeros=Tensor((100, 7), u8)), dict(y=Tensor((3, 100), bf)),
                   dict(bias=Tensor((99,), bf))):
        with pytest.raises(B.AstraError):
            B.astra_w4_linear(w, **{**fit, **change})
