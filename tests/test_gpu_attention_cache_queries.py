"""Attention over the paged cache for query rows whose dims differ widely in
size: fp32 scores whatever the range, on every path and in both formats.  The
keys are zero at the large dims, so that scores stay of ordinary size and the
small dims decide them; the bar is kv_ref.bound as for any other rows."""
import numpy as np
import pytest

from tests import kv_ref
from tests.test_gpu_attention_cache import check, env, filled, i32, on_gpu, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def zero_keys_at(cache, dims):
    """The cache with every key zero at `dims`."""
    k, v, ks, vs = cache
    if ks is None:
        k[..., dims] = 0
        return k, v, ks, vs
    code = kv_ref.unpack(k)
    code[..., dims] = 0
    return kv_ref.pack(code), v, ks, vs


def attend(env, b, cache, qb, heads, kvh, dh, ws=True, scale=None):
    ds, gu, torch = env
    batch = ds.KVBatch(i32(torch, b.q_start), i32(torch, b.kv), i32(torch, b.table), b.rows)
    out = torch.full((b.rows, heads, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    w = workspace(env, b, heads, kvh, dh, max(b.q), max(b.kv), 0, 0) if ws else None
    ds.attention_cache(gu.dev_bf16(qb).view(b.rows, heads, dh), on_gpu(env, cache), batch, out, max(b.q), max(b.kv),
                       scale=scale, workspace=w)
    torch.cuda.synchronize()
    return gu.host(out)


def reference(b, cache, qb, heads, dh, scale=None):
    return kv_ref.attend(b, kv_ref.values(cache[0], cache[2]), kv_ref.values(cache[1], cache[3]),
                         kv_ref.from_bf16_bits(qb).reshape(b.rows, heads, dh), 0, 0, dh ** -0.5 if scale is None else scale)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 16, 40])  # of 4 heads a key head: 4, 20 and 64 rows a unit, and tiles
@pytest.mark.parametrize("powers", [(8, 10, 12), (14, 16, 18, 20), (24, 31, 60, 100)])
def test_dims_far_apart(env, powers, n, dh, fp4):
    print("dims far apart", powers, n, dh, fp4, flush=True)
    heads, kvh = 8, 2
    rng = np.random.default_rng(71)
    b = kv_ref.Batch(rng, [n, n], [130, 77], 16)
    for dims in ([3], [5, 40], list(range(17, dh, 32))):
        cache = zero_keys_at(filled(rng, b, kvh, dh, fp4), dims)
        q = rng.standard_normal((b.rows, heads, dh))
        far = np.array(powers)[np.arange(b.rows * heads) % len(powers)].reshape(b.rows, heads, 1)
        q[..., dims] = np.ldexp(rng.choice([-1.0, 1.0, 1.984375], q[..., dims].shape), far)
        qb = kv_ref.to_bf16_bits(q.reshape(b.rows, -1))
        got = attend(env, b, cache, qb, heads, kvh, dh)
        check(b, got, reference(b, cache, qb, heads, dh), None)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("n", [1, 5, 40])
def test_one_row_of_many(env, n, fp4):
    """One head of one row is far apart: its own result is right, and the others' do not move."""
    heads, kvh, dh = 8, 2, 128
    rng = np.random.default_rng(72)
    b = kv_ref.Batch(rng, [n], [200], 32)
    cache = zero_keys_at(filled(rng, b, kvh, dh, fp4), [9])
    q = rng.standard_normal((b.rows, heads, dh))
    q[b.rows // 2, 3, 9] = 2.0 ** 50
    qb = kv_ref.to_bf16_bits(q.reshape(b.rows, -1))
    check(b, attend(env, b, cache, qb, heads, kvh, dh), reference(b, cache, qb, heads, dh), None)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("power", [-100, -30, 30, 100])
def test_size_of_all_dims(env, power, fp4):
    """Rows of any size, the softmax's scale making up for it."""
    heads, kvh, dh = 4, 1, 128
    for n in (1, 40):
        rng = np.random.default_rng(73)
        b = kv_ref.Batch(rng, [n], [150], 16)
        cache = filled(rng, b, kvh, dh, fp4)
        qb = kv_ref.to_bf16_bits(np.ldexp(rng.standard_normal((b.rows, heads * dh)), power))
        scale = 2.0 ** -power * dh ** -0.5
        check(b, attend(env, b, cache, qb, heads, kvh, dh, scale=scale), reference(b, cache, qb, heads, dh, scale), None)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("n", [1, 5, 40])
def test_rows_that_are_not_finite(env, n, fp4):
    """An infinity or a NaN in a row's head makes that head's output NaN, and no other."""
    heads, kvh, dh = 8, 2, 64
    rng = np.random.default_rng(74)
    b = kv_ref.Batch(rng, [n], [90], 16)
    cache = filled(rng, b, kvh, dh, fp4)
    qb = kv_ref.to_bf16_bits(rng.standard_normal((b.rows, heads * dh)))
    r = b.rows // 2
    for head, what in ((1, 0x7F80), (4, 0x7FC0), (6, 0xFF80)):
        qb[r, head * dh + 20] = what
    got = attend(env, b, cache, qb, heads, kvh, dh)
    with np.errstate(all="ignore"):
        ref = reference(b, cache, qb, heads, dh)
        check(b, got, ref, None)
    assert np.isnan(got[r, [1, 4, 6]]).all() and np.isfinite(np.delete(got[r], [1, 4, 6], 0)).all()


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("power", [-113, 113])
def test_scale_near_its_ends(env, power, fp4):
    """Scales of 2^-122 and 2^109 (of a range of 2^-126 to 2^126), the rows' size making up for them."""
    heads, kvh, dh = 4, 1, 64
    for n in (1, 40):
        rng = np.random.default_rng(75)
        b = kv_ref.Batch(rng, [n], [150], 16)
        cache = filled(rng, b, kvh, dh, fp4)
        qb = kv_ref.to_bf16_bits(np.ldexp(rng.standard_normal((b.rows, heads * dh)), power))
        scale = 2.0 ** -power * 2.0 ** -(9 if power > 0 else 4)
        check(b, attend(env, b, cache, qb, heads, kvh, dh, scale=scale), reference(b, cache, qb, heads, dh, scale), None)
