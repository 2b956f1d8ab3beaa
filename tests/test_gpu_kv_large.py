"""The cache's calls at their large ends: caches past 4 GiB in both formats,
and more sequences times key heads than a workspace has arrival counters."""
import numpy as np
import pytest

from tests import kv_ref
from tests.test_gpu_attention_cache import check, env, i32, run  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp4", [False, True])
def test_append_read_and_attend_past_32_bits(env, fp4):
    """5 GiB of keys and as many of values: pages at both ends and around 4 GiB."""
    ds, gu, torch = env
    print("past 32 bits", fp4, flush=True)
    heads, kvh, page, dh = 8, 8, 64, 128
    page_bytes = kvh * page * dh * 2 // (4 if fp4 else 1)
    n_pages = (5 << 30) // page_bytes
    rng = np.random.default_rng(91)
    b = kv_ref.Batch(rng, [130, 70], [130, 70], page)
    at4 = (4 << 30) // page_bytes
    remap = np.array([0, n_pages - 1, at4 - 1, at4, at4 + 1, n_pages - 2, 1])[:b.n_pages]
    idx = torch.from_numpy(remap).cuda()
    shape = (n_pages, kvh, page, dh // 2 if fp4 else dh)
    dtype = torch.uint8 if fp4 else torch.bfloat16
    k, v = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in "kv")
    ks, vs = ((torch.full((n_pages, kvh, dh // 32, page), 255, dtype=torch.uint8, device="cuda") for _ in "kv")
              if fp4 else (None, None))
    c = ds.KVCache(k, v, ks, vs)
    small = [np.zeros((b.n_pages, kvh, page, dh // 2), dtype=np.uint8) if fp4 else
             np.zeros((b.n_pages, kvh, page, dh), dtype=np.uint16) for _ in "kv"]
    small += [np.full((b.n_pages, kvh, dh // 32, page), 255, dtype=np.uint8) if fp4 else None for _ in "kv"]
    table = np.where(b.table >= 0, remap[np.maximum(b.table, 0)], -1)
    batch = ds.KVBatch(i32(torch, b.q_start), i32(torch, b.kv), i32(torch, table), b.rows)
    xb = kv_ref.to_bf16_bits(rng.standard_normal((b.rows, (heads + 2 * kvh) * dh)))
    q = torch.empty(b.rows, heads, dh, dtype=torch.bfloat16, device="cuda")
    ds.kv_append(c, batch, gu.dev_bf16(xb), heads, None, q)
    ko, vo = (torch.empty(b.rows, kvh, dh, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    ds.kv_read(c, batch, ko, vo)
    out = torch.empty_like(q)
    ds.attention_cache(q, c, batch, out, 130, 130)
    # single tokens over the same keys: the few-row kernel
    one = ds.KVBatch(i32(torch, [0, 1, 2]), i32(torch, b.kv), i32(torch, table), 2)
    last = [129, 199]
    o1 = torch.empty(2, heads, dh, dtype=torch.bfloat16, device="cuda")
    ds.attention_cache(q[last].contiguous(), c, one, o1, 1, 130)
    torch.cuda.synchronize()
    queries = kv_ref.append(b, *small, kv_ref.from_bf16_bits(xb), heads, kvh, None, False)
    for t, w in zip(c.tensors, small):
        if w is not None:
            got = t[idx].cpu()
            assert np.array_equal(got.numpy() if fp4 else got.view(torch.int16).numpy().view(np.uint16), w)
    vals = kv_ref.values(small[0], small[2]), kv_ref.values(small[1], small[3])
    for r, s, pos in b.row_places():
        p, slot = b.place(s, pos)
        assert np.array_equal(gu.host(ko)[r], vals[0][p, :, slot]) and np.array_equal(gu.host(vo)[r], vals[1][p, :, slot])
    ref = kv_ref.attend(b, *vals, np.stack([queries[r] for r in range(b.rows)]), 0, 0, dh ** -0.5)
    check(b, gu.host(out), ref, None)
    for i, r in enumerate(last):
        assert np.all(np.abs(gu.host(o1)[i] - ref[r][0]) <= kv_ref.bound(*ref[r]))
    # nothing else of the cache was written
    for t, empty in zip(c.tensors, (0, 0, 255, 255)):
        if t is not None:
            t[idx] = empty
            for part in t.split(1 << 12):
                assert bool((part == empty).all())


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("chunk", [1, 40])
def test_more_units_than_counters(env, chunk, fp4):
    """520 sequences on 8 key heads are 4160 units: none is split, with a workspace or without."""
    ds, gu, torch = env
    rng = np.random.default_rng(92)
    q = [1] * 519 + [chunk]
    kv = [n + int(x) for n, x in zip(q, rng.integers(0, 70, 520))]
    b = kv_ref.Batch(rng, q, kv, 16)
    assert ds.attention_cache_workspace_bytes(b.rows, 520, 8, 8, 64, chunk, max(kv)) == 0
    ws = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")
    first = run(env, b, fp4, 8, 8, 64, ws=ws)
    assert np.array_equal(run(env, b, fp4, 8, 8, 64, ws=None), first)
