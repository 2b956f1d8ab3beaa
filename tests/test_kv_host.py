"""Key/value cache: the 64-bit reference's own pins, and every refusal of the
entry points (no GPU: nothing is launched by a refused call)."""
import ctypes

import numpy as np
import pytest

import paper_2304_13541_amd as ds
from tests import kv_ref


def test_reference_fp4_pins():
    y = np.zeros((1, 32))
    y[0, :16] = [7, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.76, 0.26, -5.1, 6.9, 0, -0.0, 1.5]
    code, scale = kv_ref.fp4_encode(y)
    assert scale.tolist() == [[127]]
    assert code[0, :16].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 8, 10, 1, 15, 7, 0, 8, 3]
    for top, byte in ((7.0, 127), (np.nextafter(7.0, 8), 128), (14.0, 128), (3.5, 126), (0.0, 2), (2.0 ** -130, 2),
                      (1.4 * 2.0 ** 128, 253), (np.inf, 255), (np.nan, 255)):
        y[:] = 0
        y[0, 3] = -top
        assert kv_ref.fp4_encode(y)[1].tolist() == [[byte]], top


def test_reference_fp4_of_huge_values():
    y = np.zeros((1, 32))
    y[0, :4] = [2.0 ** 240, -(2.0 ** 130), 2.0 ** 127, 7 * 2.0 ** 127]
    code, scale = kv_ref.fp4_encode(y)
    assert scale.tolist() == [[254]] and code[0, :5].tolist() == [7, 15, 2, 7, 0]


def test_reference_fp4_is_nearest():
    rng = np.random.default_rng(5)
    y = rng.standard_normal((400, 64)) * 2.0 ** rng.integers(-20, 20, (400, 1))
    code, scale = kv_ref.fp4_encode(y)
    back = kv_ref.fp4_decode(code, scale)
    step = np.ldexp(1.0, scale.astype(int) - 127).repeat(32, -1)
    assert np.all(np.abs(back - y) <= step)  # never off by more than the scale
    for c in range(16):  # no other code is nearer
        other = kv_ref.fp4_decode(np.full_like(code, c), scale)
        assert np.all(np.abs(back - y) <= np.abs(other - y))


def test_reference_bf16_rounding():
    import torch
    rng = np.random.default_rng(6)
    x = np.concatenate((rng.standard_normal(20000) * 2.0 ** rng.integers(-140, 126, 20000), [0.0, -0.0, np.inf, 3.4e38]))
    f = x.astype(np.float32)
    want = torch.from_numpy(f).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)
    assert np.array_equal(kv_ref.to_bf16_bits(f.astype(np.float64)), want)


PTR = 0x7F0000000000  # never read: every call below is refused on the host


def cache(**kw):
    f = dict(format=0, kv_heads=2, dh=64, page_size=16, n_pages=4, k=PTR, v=PTR, k_scale=0, v_scale=0)
    f.update(kw)
    return ds._KVCache(*(f[n] or None if n in ("k", "v", "k_scale", "v_scale") else f[n] for n, _ in ds._KVCache._fields_))


def batch(**kw):
    f = dict(n_seq=1, rows=1, max_pages=2, q_start=PTR, kv_len=PTR, page_table=PTR)
    f.update(kw)
    return ds._KVBatch(*(f[n] or None if n in ("q_start", "kv_len", "page_table") else f[n] for n, _ in ds._KVBatch._fields_))


def ref(x):
    return None if x is None else ctypes.byref(x)


def append(c, b, qkv=PTR, stride=384, heads=2, cs=PTR, n=8, rot=64, pairs=0, q_out=PTR):
    return ds.lib().dstack_op_kv_append(ref(c), ref(b), qkv, stride, heads, cs, n, rot, pairs, q_out, None)


def read(c, b, k_out=PTR, v_out=PTR):
    return ds.lib().dstack_op_kv_read(ref(c), ref(b), k_out, v_out, None)


def attend(c, b, q=PTR, stride=128, heads=2, max_q=1, max_kv=32, window=0, sinks=0, scale=0.125, out=PTR, ws=None, n=0):
    return ds.lib().dstack_op_attention_cache(ref(c), ref(b), q, stride, heads, max_q, max_kv, window, sinks, scale,
                                              out, ws, n, None)


BAD_CACHE = [(dict(format=2), ds.E_UNSUPPORTED), (dict(format=-1), ds.E_UNSUPPORTED), (dict(k=0), ds.E_INVALID),
             (dict(v=0), ds.E_INVALID), (dict(format=1), ds.E_INVALID), (dict(format=1, k_scale=PTR), ds.E_INVALID),
             (dict(kv_heads=0), ds.E_INVALID), (dict(n_pages=0), ds.E_INVALID), (dict(dh=96), ds.E_UNSUPPORTED),
             (dict(dh=32), ds.E_UNSUPPORTED), (dict(page_size=0), ds.E_INVALID), (dict(page_size=8), ds.E_UNSUPPORTED),
             (dict(page_size=48), ds.E_UNSUPPORTED), (dict(page_size=2048), ds.E_UNSUPPORTED),
             (dict(kv_heads=65536), ds.E_UNSUPPORTED), (dict(n_pages=1 << 27), ds.E_UNSUPPORTED), (dict(k=PTR + 8), ds.E_INVALID), (dict(v=PTR + 2), ds.E_INVALID),
             (dict(format=1, k_scale=PTR, v_scale=PTR + 4), ds.E_INVALID)]
BAD_BATCH = [(dict(n_seq=0), ds.E_INVALID), (dict(rows=0), ds.E_INVALID), (dict(rows=-1), ds.E_INVALID),
             (dict(max_pages=0), ds.E_INVALID), (dict(q_start=0), ds.E_INVALID), (dict(kv_len=0), ds.E_INVALID),
             (dict(page_table=0), ds.E_INVALID), (dict(n_seq=65536), ds.E_UNSUPPORTED),
             (dict(max_pages=1 << 27), ds.E_UNSUPPORTED), (dict(kv_len=PTR + 2), ds.E_INVALID)]


@pytest.mark.parametrize("call", [append, read, attend])
def test_bad_cache_and_batch(call):
    assert call(None, batch()) == ds.E_INVALID and call(cache(), None) == ds.E_INVALID
    for kw, st in BAD_CACHE:
        assert call(cache(**kw), batch()) == st, kw
        assert ds.lib().dstack_last_error()
    for kw, st in BAD_BATCH:
        assert call(cache(), batch(**kw)) == st, kw


def test_append_refusals():
    for kw in (dict(qkv=None), dict(stride=383), dict(stride=-384), dict(heads=-1), dict(heads=3), dict(rot=0), dict(rot=63),
               dict(rot=66), dict(rot=-2), dict(n=0), dict(cs=None), dict(cs=None, rot=0, qkv=PTR + 1),
               dict(q_out=PTR + 1), dict(cs=PTR + 2)):
        assert append(cache(), batch(), **kw) == ds.E_INVALID, kw
    for kw in (dict(k_out=None), dict(v_out=None), dict(k_out=PTR + 1)):
        assert read(cache(), batch(), **kw) == ds.E_INVALID, kw


def test_attention_refusals():
    for kw in (dict(q=None), dict(out=None), dict(stride=127), dict(heads=0), dict(heads=3), dict(max_q=0),
               dict(max_kv=-1), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(q=PTR + 1), dict(out=PTR + 1), dict(ws=PTR + 64, n=1 << 20)):
        assert attend(cache(), batch(), **kw) == ds.E_INVALID, kw


def test_binding_refuses_other_shapes():
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)  # noqa: E731
    with pytest.raises(ValueError):
        ds.KVCache(z(2, 1, 16, 64), z(2, 1, 32, 64))
    with pytest.raises(ValueError):
        ds.KVCache(z(2, 1, 16, 64, dtype=torch.float32), z(2, 1, 16, 64, dtype=torch.float32))
    with pytest.raises(ValueError):
        ds.KVCache(z(2, 1, 64, 16).transpose(2, 3), z(2, 1, 16, 64))
    u = lambda *s: z(*s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError):
        ds.KVCache(u(2, 1, 16, 32), u(2, 1, 16, 32), u(2, 1, 16, 2), u(2, 1, 16, 2))
    with pytest.raises(ValueError):
        ds.KVCache(u(2, 1, 16, 32), u(2, 1, 16, 32), u(2, 1, 2, 16))
    i = lambda *s: z(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        ds.KVBatch(i(2), i(2), i(2, 3), 1)
    with pytest.raises(ValueError):
        ds.KVBatch(i(3).long(), i(2), i(2, 3), 1)
    c = ds.KVCache(z(2, 1, 16, 64), z(2, 1, 16, 64))
    b = ds.KVBatch(i(3), i(2), i(2, 3), 4)
    with pytest.raises(ValueError):
        ds.kv_append(c, b, z(4, 128), 1, None, z(4, 1, 64))  # too narrow
    with pytest.raises(ValueError):
        ds.kv_append(c, b, z(3, 192), 1, None, z(4, 1, 64))  # too few rows
    with pytest.raises(ValueError):
        ds.kv_read(c, b, z(4, 1, 32), z(4, 1, 64))
    with pytest.raises(ValueError):
        ds.attention_cache(z(4, 1, 64), c, b, z(4, 1, 128)[..., ::2], 2, 32)
    with pytest.raises(ValueError):
        ds.attention_cache(z(4, 1, 64).float(), c, b, z(4, 1, 64), 2, 32)


def test_binding_refuses_other_devices():
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)  # noqa: E731
    c = ds.KVCache(z(2, 1, 16, 64), z(2, 1, 16, 64))
    b = ds.KVBatch(*(z(*s, dtype=torch.int32) for s in ((2,), (1,), (1, 3))), 4)
    calls = (lambda: ds.kv_append(c, b, z(4, 192), 1, None, z(4, 1, 64)), lambda: ds.kv_read(c, b, z(4, 1, 64), z(4, 1, 64)),
             lambda: ds.attention_cache(z(4, 1, 64), c, b, z(4, 1, 64), 2, 32))
    for call in calls:
        with pytest.raises(ValueError, match="one GPU"):  # host memory
            call()
    c.device = 1
    for call in calls:
        with pytest.raises(ValueError, match="one GPU"):  # the batch elsewhere
            call()
    b.device = 1

    class Stream:
        cuda_stream, device_index = 0, 0
    st = Stream()
    calls = (lambda: ds.kv_append(c, b, z(4, 192), 1, None, z(4, 1, 64), stream=st),
             lambda: ds.kv_read(c, b, z(4, 1, 64), z(4, 1, 64), st),
             lambda: ds.attention_cache(z(4, 1, 64), c, b, z(4, 1, 64), 2, 32, stream=st))
    for call in calls:
        with pytest.raises(ValueError, match="stream"):
            call()
    st.device_index = 1
    for call in calls:
        with pytest.raises(ValueError, match="not on the cache's GPU"):  # the rows elsewhere
            call()


def test_more_threads_than_a_launch_has():
    big = batch(rows=1 << 29)
    assert append(cache(kv_heads=8), big, stride=1152) == ds.E_UNSUPPORTED
    assert append(cache(kv_heads=8), big, stride=1153) == ds.E_UNSUPPORTED
    assert read(cache(kv_heads=8), big) == ds.E_UNSUPPORTED
    assert attend(cache(), batch(rows=1 << 30), max_q=1 << 30) == ds.E_UNSUPPORTED
    assert attend(cache(kv_heads=512), batch(n_seq=65535, rows=65535), heads=512, stride=512 * 64, max_q=65535) == ds.E_UNSUPPORTED


def test_workspace_bytes_of_bad_sizes():
    assert ds.attention_cache_workspace_bytes(0, 1, 1, 1, 64, 1, 10) == 0
    assert ds.attention_cache_workspace_bytes(1, 1, 3, 2, 64, 1, 10) == 0
    assert ds.attention_cache_workspace_bytes(1, 1, -1, 1, 64, 1, 10) == 0


def test_integers_past_32_bits():
    """A window of 2^32 + 5 is no window of 5: refused, not taken modulo 2^32."""
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)  # noqa: E731
    tensors = [z(*s, dtype=torch.int32) for s in ((2,), (1,), (1, 3))]
    with pytest.raises(ValueError, match="below 2.31"):
        ds.KVBatch(*tensors, (1 << 32) + 4)
    c, b = ds.KVCache(z(2, 1, 16, 64), z(2, 1, 16, 64)), ds.KVBatch(*tensors, 4)
    for kw in (dict(max_q=(1 << 32) + 1), dict(max_kv=1 << 31), dict(window=(1 << 32) + 5), dict(sinks=1 << 40),
               dict(window=-(1 << 32) + 5)):
        with pytest.raises(ValueError, match="below 2.31"):
            ds.attention_cache(z(4, 1, 64), c, b, z(4, 1, 64), **{**dict(max_q=2, max_kv=32), **kw})
        sizes = dict(rows=4, n_seq=1, heads=1, kv_heads=1, dh=64, max_q=2, max_kv=32)
        with pytest.raises(ValueError, match="below 2.31"):
            ds.attention_cache_workspace_bytes(**{**sizes, **kw})


def test_scale_out_of_range():
    """Scales whose product with log2 e fp32 does not hold are refused (they were taken as 1e-37 and 3e38)."""
    for scale in (2.0 ** -127, -1e-40, 1e-45, 2.0 ** 126 * 1.01, -3e38):
        assert attend(cache(), batch(), scale=scale) == ds.E_INVALID, scale
