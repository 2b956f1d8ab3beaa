"""Infinities among values that rows see, at keys whose weight is far below
what fp32 holds: the outputs they reach are infinite (NaN where infinities of
both signs meet), however the keys are split and wherever in a tile they lie."""
import numpy as np
import pytest

from tests import kv_ref
from tests.test_gpu_attention_cache import check, env, filled  # noqa: F401
from tests.test_gpu_attention_cache_queries import attend, reference

pytestmark = pytest.mark.gpu

HEADS, KVH, DH = 8, 2, 64


def put(cache, place, fp4, score, dim, sign):
    """Key at `place`: `score` in dim 0 and zeros; value: an infinity at `dim`, zeros beside it."""
    k, v, ks, vs = cache
    p, s = place
    row = np.zeros((KVH, DH))
    row[:, 0] = score
    if fp4:
        code, scale = kv_ref.fp4_encode(row)
        k[p, :, s], ks[p, :, :, s] = kv_ref.pack(code), scale
        code = np.zeros((KVH, DH), dtype=np.uint8)
        code[:, dim] = 7 if sign > 0 else 14  # 6 * 2^127, -4 * 2^126: past bf16
        v[p, :, s], vs[p, :, :, s] = kv_ref.pack(code), 254 if sign > 0 else 253
    else:
        k[p, :, s] = kv_ref.to_bf16_bits(row)
        v[p, :, s] = 0
        v[p, :, s, dim] = 0x7F80 if sign > 0 else 0xFF80


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("n", [1, 5, 16, 40])
@pytest.mark.parametrize("kv", [70, 1500])
def test_infinity_of_little_weight(env, kv, n, fp4):
    """Scores 240 below the others' (a weight of 2^-346): near both ends of the keys and amid them."""
    print("infinity of little weight", kv, n, fp4, flush=True)
    rng = np.random.default_rng(81)
    b = kv_ref.Batch(rng, [n], [kv], 16)
    q = rng.standard_normal((b.rows, HEADS, DH))
    q[..., 0] = 16.0
    qb = kv_ref.to_bf16_bits(q.reshape(b.rows, -1))
    for at in ([(2, 5, 1)], [(kv - n - 1, 6, -1)], [(kv // 2, 7, 1), (kv // 2 + 1, 8, -1)],
               [(3, 9, 1), (kv - n - 3, 9, -1), (kv // 3, 40, 1)]):
        cache = filled(rng, b, KVH, DH, fp4)
        k, ks = cache[0], cache[2]
        if fp4:  # dim 0 of the others counts nothing
            code = kv_ref.unpack(k)
            code[..., 0] = 0
            cache = (kv_ref.pack(code),) + cache[1:]
        else:
            k[..., 0] = np.where(k[..., 0] == 0x7FC0, k[..., 0], 0)
        for j, dim, sign in at:
            put(cache, b.place(0, j), fp4, -120.0, dim, sign)
        with np.errstate(all="ignore"):
            ref = reference(b, cache, qb, HEADS, DH)
            for ws in (True, False):
                got = attend(env, b, cache, qb, HEADS, KVH, DH, ws=ws)
                check(b, got, ref, None)
                for j, dim, _ in at:  # in every row from the key's own position on
                    assert not np.isfinite(got[max(0, j - (kv - n)):, :, dim]).any()


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("n", [1, 40])
def test_infinity_before_larger_scores(env, n, fp4):
    """The infinity's key has the largest score of its part; parts after it have scores 240 above."""
    rng = np.random.default_rng(82)
    kv = 1500
    b = kv_ref.Batch(rng, [n], [kv], 16)
    q = rng.standard_normal((b.rows, HEADS, DH))
    q[..., 0] = 16.0
    qb = kv_ref.to_bf16_bits(q.reshape(b.rows, -1))
    cache = filled(rng, b, KVH, DH, fp4)
    rows = np.zeros((KVH, DH))
    for j in range(kv):  # scores 0 up to the 1000th key, then 240
        p, s = b.place(0, j)
        rows[:, 0] = 0.0 if j < 1000 else 120.0
        if fp4:
            code, scale = kv_ref.fp4_encode(rows)
            cache[0][p, :, s], cache[2][p, :, :, s] = kv_ref.pack(code), scale
        else:
            cache[0][p, :, s] = kv_ref.to_bf16_bits(rows)
    put(cache, b.place(0, 130), fp4, 0.0, 11, 1)
    with np.errstate(all="ignore"):
        ref = reference(b, cache, qb, HEADS, DH)
        for ws in (True, False):
            got = attend(env, b, cache, qb, HEADS, KVH, DH, ws=ws)
            check(b, got, ref, None)
            assert np.all(got[:, :, 11] == np.inf)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("power", [-100, 100])
def test_values_of_any_size(env, power, fp4):
    """Finite values of any size up to what the sums hold stay finite, split or not."""
    for n, kv in ((1, 1500), (40, 400)):
        rng = np.random.default_rng(83)
        b = kv_ref.Batch(rng, [n], [kv], 16)
        k, v, ks, vs = filled(rng, b, KVH, DH, fp4, stale=False)
        if fp4:
            vs = (vs.astype(int) + power).astype(np.uint8)
        else:
            v = kv_ref.to_bf16_bits(np.ldexp(kv_ref.from_bf16_bits(v), power))
        qb = kv_ref.to_bf16_bits(rng.standard_normal((b.rows, HEADS * DH)))
        for ws in (True, False):
            check(b, attend(env, b, (k, v, ks, vs), qb, HEADS, KVH, DH, ws=ws), reference(b, (k, v, ks, vs), qb, HEADS, DH), None)
