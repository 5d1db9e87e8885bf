"""hils_cache_reserve, _fork, _free and _compact against their plain statement (tests/pages_oracle.py): whole
numbers and copied bytes, so everything has to be equal."""
import numpy as np
import pytest
import torch

from tests import pages_oracle as O

pytestmark = pytest.mark.gpu


def hils_():
    from paper_2607_02980_amd import hils

    return hils


def params(B, L, N=1):
    return hils_().Params(B=B, Hq=4, Hkv=2, N=N, L=L, d=64, topk=2, window=64)


def dev(x, dtype=torch.int32):
    return None if x is None else torch.as_tensor(np.asarray(x)).to("cuda", dtype)


def same(got, ref, what=""):
    for i, (x, y) in enumerate(zip(got, ref)):
        x = x.cpu().numpy()
        assert x.shape == np.shape(y) and np.array_equal(x, y), f"{what} output {i}: {x} instead of {y}"


def state(p, rng, lens, spare, share=0.5):
    """Sequences that share a random beginning with an earlier one (to the end of it, sometimes), pages anywhere;
    entries past a length hold anything."""
    C = p.L // O.S
    rows, count = [], 0
    for b in range(p.B):
        n = O.chunks(lens[b])
        row = []
        if b and rng.random() < share:
            u = int(rng.integers(b))
            if O.chunks(lens[u]) >= n and rng.random() < 0.5:
                row = rows[u][:n]
            else:
                row = rows[u][:int(rng.integers(0, min(n, O.chunks(lens[u])) + 1))]
        row = row + list(range(count, count + n - len(row)))
        count = max([count] + [x + 1 for x in row])
        rows.append(row)
    P = count + spare
    perm = rng.permutation(P)
    table = rng.integers(-5, P + 5, (p.B, C)).astype(np.int32)
    refs = np.zeros(P, np.int32)
    for b, row in enumerate(rows):
        table[b, :len(row)] = perm[row]
        np.add.at(refs, perm[row], 1)
    free = np.flatnonzero(refs == 0)
    refs[free[::3]] = -1  # (0 or less is free)
    return table, refs


def pool_set(P, rng, many=0):
    """Pools of several types and page sizes, one of them of an odd number of bytes at an odd address."""
    shapes = [((2, 64, 64), torch.bfloat16), ((2, 64, 64), torch.float32), ((4, 64), torch.bfloat16), ((4,), torch.float32),
              ((2, 64, 64), torch.float8_e4m3fn), ((3,), torch.uint8), ((40000,), torch.uint8)] + [((5,), torch.int16)] * many
    out = []
    for i, (shape, dt) in enumerate(shapes):
        n = P * int(np.prod(shape)) * dt.itemsize
        raw = torch.as_tensor(rng.integers(0, 256, n + 1).astype(np.uint8)).cuda()
        t = raw[1:] if dt == torch.uint8 and shape == (3,) else raw[:n]
        out.append((t.view(P, *shape) if dt == torch.uint8 else t.view(dt).view(P, *shape)))
    return out


def bytes_of(pools):
    return [x.contiguous().view(torch.uint8).reshape(x.shape[0], -1).cpu().numpy() for x in pools]


def check_pools(pools, before, ref):
    after = bytes_of(pools)
    for i, (x, y) in enumerate(zip(after, ref)):
        assert np.array_equal(x, y), f"pool {i}"


CASES = [  # B, L, N, lens, new, spare
    (1, 64, 1, [1], [1], 1),
    (1, 64, 1, [64], [0], 1),
    (3, 256, 256, [256, 100, 0], [256, 3, 0], 20),
    (5, 640, 70, [640, 65, 64, 130, 70], [70, 1, 64, 66, 70], 40),
    (7, 1024, 5, None, None, 60),
    (40, 2048, 200, None, None, 500),
]


def lens_of(case, seed):
    B, L, N, lens, new, spare = case
    r = np.random.default_rng(seed)
    if lens is None:
        lens = r.integers(0, L + 1, B)
        new = r.integers(0, N + 1, B)
    return list(map(int, lens)), list(map(int, new))


@pytest.mark.parametrize("seed", [0, 1, 2])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"B{c[0]}_L{c[1]}_N{c[2]}")
@pytest.mark.parametrize("in_place", [False, True])
def test_reserve(case, seed, in_place):
    hils, r = hils_(), np.random.default_rng(seed + 10)
    p = params(*case[:3])
    lens, new = lens_of(case, seed)
    old = [a - min(m, a) for a, m in zip(lens, new)]
    table, refs = state(p, r, old, case[5])
    pools = pool_set(len(refs), r)
    before = bytes_of(pools)
    after = [x.copy() for x in before]
    ref = O.reserve(p, table, refs, after, lens, new)
    assert ref[3][0] == ref[3][1]
    t, n = dev(table), dev(refs)
    kw = dict(table_out=t, refs_out=n) if in_place else {}
    got = hils.hils_cache_reserve(p, t, n, pools, dev(lens), dev(new), **kw)
    same(got, ref)
    check_pools(pools, before, after)
    if not in_place:
        same((t, n), (table, refs), "inputs")


def test_reserve_all_writers_of_a_page():
    """Four beams of one sequence: the first keeps the begun page if all who have it write, else all take copies."""
    hils = hils_()
    p = params(4, 256)
    table = np.int32([[3, 5, -1, -1]] * 4)
    for extra in (0, 1):
        refs = np.int32([0, 0, 0, 4, 0, 4 + extra, 0, 0, 0, 0])
        pool = torch.arange(10, device="cuda", dtype=torch.float32).view(10, 1)
        got = hils.hils_cache_reserve(p, dev(table), dev(refs), [pool], dev([101] * 4))
        ref = O.reserve(p, table, refs, [np.arange(10.0)], [101] * 4)
        same(got, ref)
        given = [0, 1, 2, 4][:3 + extra]
        assert got[0][:, 1].tolist() == ([] if extra else [5]) + given and got[1][5].item() == 1
        assert pool.flatten().tolist() == [5 if i in given else i for i in range(10)]


def test_reserve_without_enough_pages_does_nothing():
    hils = hils_()
    p = params(3, 640, 200)
    r = np.random.default_rng(3)
    lens, new = [300, 200, 210], [200, 200, 10]
    table, refs = state(p, r, [100, 0, 200], 4, share=0)
    pools = pool_set(len(refs), r)
    before = bytes_of(pools)
    got = hils.hils_cache_reserve(p, dev(table), dev(refs), pools, dev(lens), dev(new))
    need = 3 + 4 + 0
    same(got, (table, refs, np.full((3, 2), -1), [need, 4]))
    check_pools(pools, before, before)
    same(got, O.reserve(p, table, refs, before, lens, new))


def test_reserve_defaults_and_clamping():
    hils = hils_()
    p = params(2, 256, 100)
    refs = np.zeros(9, np.int32)
    got = hils.hils_cache_reserve(p, dev(np.full((2, 4), 99)), dev(refs))  # lengths L, N new tokens each: entries of no page
    same(got, O.reserve(p, np.full((2, 4), 99), refs, []))
    assert got[3].tolist() == [4, 4]
    got = hils.hils_cache_reserve(p, dev(np.full((2, 4), -1)), dev(refs), seqlens=dev([1000, -3]), newlens=dev([1000, 7]))
    same(got, O.reserve(p, np.full((2, 4), -1), refs, [], [1000, -3], [1000, 7]))


@pytest.mark.parametrize("P,B", [(16384, 3), (16385, 3), (70001, 1100), (200000, 2500)])
def test_reserve_large_pools_and_batches(P, B):
    """Free pages far into the pool, more sequences than a workgroup has threads; pages of few bytes."""
    hils, r = hils_(), np.random.default_rng(P)
    p = params(B, 64 * 40, 200)
    lens = r.integers(0, p.L + 1, B)
    new = r.integers(0, 201, B)
    refs = np.ones(P, np.int32)
    refs[r.choice(P, 6 * B, replace=False)] = 0
    refs[-1] = 0
    used = np.flatnonzero(refs > 0)
    table = r.choice(used, (B, 40)).astype(np.int32)
    refs[used] = np.maximum(1, np.bincount(table[:, :20].ravel(), minlength=P)[used])
    pool = torch.arange(P, device="cuda", dtype=torch.int64).view(P, 1)
    after = [np.arange(P)[:, None]]
    ref = O.reserve(p, table, refs, after, lens, new)
    got = hils.hils_cache_reserve(p, dev(table), dev(refs), [pool], dev(lens), dev(new))
    assert ref[3][0] == ref[3][1] > 1
    same(got, ref)
    assert np.array_equal(pool.cpu().numpy(), after[0])


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("B,L,rows", [(1, 64, 1), (5, 640, 9), (64, 4096, 3), (3, 64 * 3000, 7)])
def test_fork(B, L, rows, seed):
    hils, r = hils_(), np.random.default_rng(seed)
    p = params(B, L)
    lens = r.integers(0, L + 1, B)
    table, refs = state(p, r, lens, 20)
    table[0, 0] = [-7, len(refs)][seed]  # an entry of no page
    parent = r.integers(-1, B, rows)
    if rows > 5:
        parent[:3] = [-2 ** 31, 2 ** 31 - 1, B]
        parent[3:5] = B - 1
    t, n, a = dev(table), dev(refs), dev(lens)
    ref = O.fork(p, parent, table, refs, lens)
    same(hils.hils_cache_fork(p, dev(parent), t, n, a), ref)
    same((t, n, a), (table, refs, lens), "inputs")
    got = hils.hils_cache_fork(p, dev(parent), t, n, a, refs_out=n)  # the counts in place
    same(got, ref)
    assert got[2] is n
    same(hils.hils_cache_fork(p, dev(parent), t, dev(refs)), O.fork(p, parent, table, refs))


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("B,L", [(1, 64), (6, 640), (70, 4096), (2, 64 * 3000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_free(B, L, seed, in_place):
    hils, r = hils_(), np.random.default_rng(seed)
    p = params(B, L)
    lens = r.integers(0, L + 1, B)
    table, refs = state(p, r, lens, 20)
    table[0, 0] = [-7, len(refs)][seed]
    keep = np.where(r.random(B) < 0.3, lens, r.integers(-3, L + 9, B))
    t, n, a = dev(table), dev(refs), dev(lens)
    kw = dict(table_out=t, seqlens_out=a, refs_out=n) if in_place else {}
    same(hils.hils_cache_free(p, dev(keep), t, n, a, **kw), O.free(p, keep, table, refs, lens))
    if not in_place:
        same((t, n, a), (table, refs, lens), "inputs")
        pages = r.integers(-2, len(refs) + 2, (B, 5))  # listed pages: of none, the same twice
        count = r.integers(-1, 8, B)
        same(hils.hils_cache_free(p, dev(keep), t, n, a, dev(pages), dev(count)), O.free(p, keep, table, refs, lens, pages, count))
        same(hils.hils_cache_free(p, dev(lens), t, n, a, dev(pages)), O.free(p, lens, table, refs, lens, pages))
        same(hils.hils_cache_free(p, dev(keep), t, n), O.free(p, keep, table, refs))


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("B,L,spare,many", [(1, 64, 0, 0), (1, 64, 1, 0), (5, 640, 30, 0), (9, 2048, 7, 30)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compact(B, L, spare, many, seed, in_place):
    hils, r = hils_(), np.random.default_rng(seed + 5)
    p = params(B, L)
    lens = r.integers(1, L + 1, B)
    table, refs = state(p, r, lens, spare)
    pools = pool_set(len(refs), r, many)  # (more than one launch of copies)
    before = bytes_of(pools)
    after = [x.copy() for x in before]
    ref = O.compact(p, table, refs, after, lens)
    t, n = dev(table), dev(refs)
    kw = dict(table_out=t, refs_out=n) if in_place else {}
    got = hils.hils_cache_compact(p, t, n, pools, dev(lens), **kw)
    if in_place:  # (counts below 0, of pages that were free, stay)
        same((got[1].clamp(min=0),), (ref[1],))
        got = got[:1] + (got[1].clamp(min=0),) + got[2:]
    same(got, ref)
    check_pools(pools, before, after)
    used = int(ref[4][0])
    assert (got[1][:used] > 0).all() and (got[1][used:] <= 0).all()


@pytest.mark.parametrize("P,used", [(1, 0), (1, 1), (2, 1), (16383, 9000), (16385, 16384), (70001, 35000), (70001, 0), (70001, 70001)])
def test_compact_pools_of_any_size(P, used):
    hils, r = hils_(), np.random.default_rng(P)
    p = params(1, 64 * max(1, used))
    pages = r.permutation(P)[:used]
    refs = np.zeros(P, np.int32)
    refs[pages] = r.integers(1, 5, used)
    table = pages[None].astype(np.int32) if used else np.full((1, 1), -1, np.int32)
    pool = torch.arange(P, device="cuda", dtype=torch.int64).view(P, 1)
    after = [np.arange(P)[:, None]]
    lens = [64 * used]
    ref = O.compact(p, table, refs, after, lens)
    same(hils.hils_cache_compact(p, dev(table), dev(refs), [pool], dev(lens)), ref)
    assert np.array_equal(pool.cpu().numpy(), after[0])


def test_no_pools_and_graph_replays():
    """All four captured into one graph and replayed on changing inputs, beside eager work."""
    hils, r = hils_(), np.random.default_rng(9)
    p = params(6, 1024, 90)
    side = torch.cuda.Stream()
    lens = [500, 64, 1000, 333, 90, 128]
    fill = [state(p, r, [a - 90 if a > 90 else 0 for a in lens], 80) for _ in range(3)]
    P = max(len(x[1]) for x in fill)
    fill = [(t, np.concatenate([n, np.zeros(P - len(n), np.int32)])) for t, n in fill]
    table, refs, ln = dev(fill[0][0]), dev(fill[0][1]), dev(lens)
    parent, keep = dev([0, 0, 3, -1, 5, 2]), dev([100, 1000, 0, 64, 65, 200])
    pool = torch.zeros((P, 3), device="cuda", dtype=torch.int32)

    def step():
        a = hils.hils_cache_reserve(p, table, refs, [pool], ln)
        b = hils.hils_cache_fork(p, parent, a[0], a[1], ln)
        c = hils.hils_cache_free(p, keep, b[0], b[2], b[1])
        return a + b + c + hils.hils_cache_compact(p, c[0], c[2], [pool], c[1])

    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step()
    for t, n in fill * 2:
        table.copy_(dev(t)), refs.copy_(dev(n)), pool.copy_(torch.arange(3 * P, device="cuda").view(P, 3))
        graph.replay()
        torch.cuda.synchronize()
        data = [np.arange(3 * P).reshape(P, 3)]
        a = O.reserve(p, t, n, data, lens)
        b = O.fork(p, [0, 0, 3, -1, 5, 2], a[0], a[1], lens)
        c = O.free(p, [100, 1000, 0, 64, 65, 200], b[0], b[2], b[1])
        same(out, a + b + c + O.compact(p, c[0], c[2], data, c[1]))
        assert np.array_equal(pool.cpu().numpy(), data[0])
        assert hils.hils_cache_reserve(p, table, refs, seqlens=ln)[3].tolist() == a[3].tolist()  # eager work between replays
