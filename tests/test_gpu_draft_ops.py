"""The speculative decoding step's operators on the GPU against their 64-bit definitions (oracle/draft.py).

Tolerances count roundings of half a step: 2^-8 of the value for bf16, 2^-24 for fp32.

* rope_append: the last rounding to bf16, 2^-8 |ref|; before it fp32.  A rotated
  value is two products and a sum of its pair, the products' factors carry the
  norm's roundings (a sum of hd <= 128 squares in at most 128 steps of which the
  root halves the effect, the root and three products): together below (64 + 8) *
  2^-24 < 2^-17 of |a| + |b|.  Values of v and rows without norm that only round
  are held to the first part alone.
* attn_tree: 2^-8 |ref| of the last rounding, and 2^-14 max |v| for the softmax
  weights, of which 2^-16 is the rest behind the pair hi + lo that enters the matrix
  cores and the others are the fp32 scores' (|z| <= 32 in these cases: 2^-24 * 32
  times the few roundings of a sum of 128, within 2^-16) and the sums'.
* sample: tokens are equal; prob rounds once to fp32 (2^-24 of it) from weights and
  sums of relative error 2^-35 (half a step of 2^-34 next to 1), of which those below
  e^-32 < 2^-46 of the largest may be missing: 2^-24 prob + 2^-28 with 2^18 of them.
* kv_move and whatever is to be left alone: equal bit for bit.
"""

import numpy as np
import pytest

from oracle import bf16_bits_to_f64
from oracle import draft as D
from paper_2411_03519_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

EPS = 1e-5
NAN_BITS = np.array([0x7FC0, 0xFFC1, 0x7F80, 0xFF80], np.uint16)


@pytest.fixture(scope="module")
def metro():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2411_03519_amd import metro as m
    return m


def bits(x):
    return synth.f32_to_bf16_bits(np.asarray(x, np.float32))


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def ints(a):
    return dev(np.asarray(a, np.int32))


def host(t):
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def empty_bits(n):
    """n bf16 values that no result would hold."""
    return torch.full((n,), 0x7FA5, dtype=torch.int16, device="cuda")


def rope_table(n_pos, hd, base=500000.0):
    angle = np.arange(n_pos)[:, None] * base ** (-2.0 * np.arange(hd // 2) / hd)
    return np.stack([np.cos(angle), np.sin(angle)], axis=2).astype(np.float32)


# --- rope_append -----------------------------------------------------------------


def append_case(metro, rng, nq, nkv, hd, pos, slot, n_pages, half, q_norm, k_norm, extra=0, n_pos=300, size=1.0):
    T, width = len(pos), (nq + 2 * nkv) * hd
    y = (size * rng.standard_normal((T, width + extra))).astype(np.float32)
    y[:, width:] = np.nan
    yb = bits(y)
    if half:
        y = bf16_bits_to_f64(yb)
    rope = rope_table(n_pos, hd)
    gains = [bits(1 + 0.1 * rng.standard_normal(hd)) if on else None for on in (q_norm, k_norm)]
    pool = rng.choice(NAN_BITS, size=(n_pages, 2, nkv, 16 * hd))
    kv, q = dev(pool), empty_bits(T * nq * hd)
    metro.op_rope_append(dev(yb).view(torch.bfloat16) if half else dev(y), T, nq, nkv, hd, dev(rope), n_pos, ints(pos), ints(slot), q, kv, n_pages,
                         q_gain=None if gains[0] is None else dev(gains[0]), k_gain=None if gains[1] is None else dev(gains[1]),
                         eps=EPS, ld=width + extra)
    want = D.rope_rows(y[:, :width], nq, nkv, hd, *[None if g is None else bf16_bits_to_f64(g) for g in gains], EPS, rope, pos)
    heads = np.abs(np.asarray(y[:, :width], np.float64)).reshape(T, -1, hd)
    pair = heads + np.roll(heads, hd // 2, axis=2)
    for part, gain in ((pair[:, :nq], gains[0]), (pair[:, nq:nq + nkv], gains[1])):
        if gain is not None:  # |a| + |b| behind the norm, gains at most 2
            part *= 2.0 / np.sqrt(np.mean(np.asarray(heads[:, :nq] if part.shape[1] == nq else heads[:, nq:nq + nkv]) ** 2, axis=2,
                                          keepdims=True) + EPS)
    tol = [2.0 ** -17 * pair[:, :nq], 2.0 ** -17 * pair[:, nq:nq + nkv], 0.0]

    def close(got, ref, t, what):
        bad = ~(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + t) & ~(np.isnan(got) & np.isnan(ref))
        assert not bad.any(), (what, np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])

    close(bf16_bits_to_f64(host(q)).reshape(T, nq, hd), want[0], tol[0], "q")
    got, left = host(kv).reshape(pool.shape), pool.copy()
    places = D.tile_places(hd)
    for t in range(T):
        if not 0 <= slot[t] < 16 * n_pages:
            continue
        p, o = slot[t] // 16, slot[t] % 16
        for c in range(2):
            tt = tol[1][t] if c == 0 else 0.0
            close(bf16_bits_to_f64(got[p, c][:, places[c][o]]), want[1 + c][t], tt, ("cache", c, t))
            left[p, c][:, places[c][o]] = got[p, c][:, places[c][o]]
    np.testing.assert_array_equal(got, left)


def runs(rng, lens, n_pages):
    """Slots and positions of sequences' consecutive tokens over scattered pages, from any place in a page."""
    ids, pos, slot, at = rng.permutation(n_pages), [], [], 0
    for n in lens:
        first = int(rng.integers(0, 200))
        o = first % 16 + np.arange(n)
        slot += list(ids[at + o // 16] * 16 + o % 16)
        pos += list(first + np.arange(n))
        at += (first % 16 + n + 15) // 16
    return np.array(pos), np.array(slot)


HEADS = [(8, 4, 64), (4, 4, 128), (8, 1, 128), (32, 8, 128), (10, 5, 64), (1, 1, 64)]


@pytest.mark.parametrize("nq,nkv,hd", HEADS)
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("norms", [(False, False), (True, True), (True, False)])
def test_append(metro, nq, nkv, hd, half, norms):
    rng = np.random.default_rng([nq, nkv, hd, half, *norms])
    for lens in ([1], [1, 1, 1], [3, 16, 17, 1, 40], [64], [5, 5, 5, 5]):
        pos, slot = runs(rng, lens, 40)
        append_case(metro, rng, nq, nkv, hd, pos, slot, 40, half, *norms)


@pytest.mark.parametrize("hd", [64, 128])
def test_append_slots_in_any_order(metro, hd):
    """Rows of one page in any order, slots outside the cache, positions outside the table, a row stride with NaN behind the heads."""
    rng = np.random.default_rng(hd)
    slot = rng.permutation(16 * 6)[:70].copy()
    pos = rng.integers(0, 300, 70)
    slot[[3, 20, 21, 69]] = [-1, 16 * 6, 2 ** 31 - 1, -2 ** 31]
    pos[[5, 33]] = [-1, 300]
    for half in (False, True):
        append_case(metro, rng, 8, 2, hd, pos, slot, 6, half, True, True, extra=24)
    append_case(metro, rng, 8, 2, hd, np.arange(32), np.arange(32)[::-1].copy(), 2, False, False, True)
    append_case(metro, rng, 8, 2, hd, np.arange(32), np.full(32, -1), 2, False, True, True)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("half", [False, True])
def test_append_norm_of_heads_whose_squares_pass_fp32(metro, hd, half):
    """Such a head comes out as 0 (|y| up to 1e18 does not: 128 of their squares are below 2^128), its values as they are."""
    rng = np.random.default_rng([hd, half])
    nq, nkv, T = 4, 2, 9
    append_case(metro, rng, nq, nkv, hd, np.arange(T), np.arange(T), 1, half, True, True, size=2e17)
    y = (rng.standard_normal((T, nq + 2 * nkv, hd))).astype(np.float32)
    y[:, 1] = y[:, nq] = 1e25
    yb, gain = bits(y), dev(bits(np.ones(hd)))
    kv, q = dev(np.zeros(2 * nkv * 16 * hd, np.uint16)), empty_bits(T * nq * hd)
    metro.op_rope_append(dev(yb).view(torch.bfloat16) if half else dev(y), T, nq, nkv, hd, dev(rope_table(T, hd)), T, ints(np.arange(T)),
                         ints(np.arange(T)), q, kv, 1, q_gain=gain, k_gain=gain, eps=EPS)
    q = bf16_bits_to_f64(host(q)).reshape(T, nq, hd)
    k = bf16_bits_to_f64(host(kv)).reshape(2, nkv, 16 * hd)[0][:, D.tile_places(hd)[0][:T]]
    assert (q[:, 1] == 0).all() and (k[0] == 0).all()
    for x in (q[:, 0], q[:, 2], q[:, 3], k[1]):
        assert np.isfinite(x).all() and (x != 0).any(axis=1).all()


def test_append_norm_of_small_and_large_rows(metro):
    rng = np.random.default_rng(8)
    for size in (0.0, 1e-6, 1e6, 1e15):
        append_case(metro, rng, 4, 2, 64, np.arange(5), np.arange(5) + 3, 2, False, True, True, size=size)


# --- attn_tree -------------------------------------------------------------------


def random_tree(rng, n):
    see = np.eye(n, dtype=bool)
    for r in range(1, n):
        see[r] |= see[int(rng.integers(max(0, r - 5), r))]
    return see


def pack_mask(seen, max_q):
    ldm = -(-max_q // 32)
    b = np.zeros((sum(len(m) for m in seen), 32 * ldm), np.uint8)
    at = 0
    for m in seen:
        b[at:at + len(m), :m.shape[1]] = m
        at += len(m)
    return np.packbits(b, axis=1, bitorder="little").view(np.int32), ldm


def tree_pool(rng, K, V, nkv, hd, spare=5):
    """The sequences' pages scattered over a pool whose other slots hold NaN and Inf."""
    need = [-(-len(k) // 16) for k in K]
    n_pages = sum(need) + spare
    ids, places = rng.permutation(n_pages), D.tile_places(hd)
    pool = rng.choice(NAN_BITS, size=(n_pages, 2, nkv, 16 * hd))
    tables, at = np.full((len(K), max(need)), -7, np.int32), 0
    for i, n in enumerate(need):
        tables[i, :n] = ids[at:at + n]
        at += n
        for c, x in enumerate((K[i], V[i])):
            for t in range(len(x)):
                pool[tables[i, t // 16], c][:, places[c][t % 16]] = x[t]
    return pool, tables


def tree_case(metro, rng, G, nkv, hd, ctxs, ns, seen=None, chain=False, scale=1.0, ws=True, K=None, V=None, max_q=None,
              max_keys=None, slack=0.0):
    nq, rows = G * nkv, sum(ns)
    if seen is None:
        seen = [np.tril(np.ones((n, n), bool)) if chain else random_tree(rng, n) for n in ns]
    q = bits(scale * rng.standard_normal((rows, nq, hd)))
    K = K or [bits(rng.standard_normal((c + n, nkv, hd))) for c, n in zip(ctxs, ns)]
    V = V or [bits(rng.standard_normal((c + n, nkv, hd))) for c, n in zip(ctxs, ns)]
    pool, tables = tree_pool(rng, K, V, nkv, hd)
    max_q, max_keys = max_q or max(ns), max_keys or max(c + n for c, n in zip(ctxs, ns))
    mask, ldm = pack_mask(seen, max_q)
    if not chain:  # bits behind an item's own queries say nothing
        at = 0
        for n in ns:
            for w in range(ldm):
                tail = 0xFFFFFFFF << min(max(n - 32 * w, 0), 32) & 0xFFFFFFFF
                mask[at:at + n, w] = (mask[at:at + n, w].astype(np.int64) | tail).astype(np.uint32).view(np.int32)
            at += n
    cu = np.concatenate([[0], np.cumsum(ns)])
    out = empty_bits(rows * nq * hd)
    n_ws = metro.op_attn_tree_workspace(nq, nkv, hd, len(ns), rows, max_q, max_keys) if ws is True else ws
    wsp = torch.full((max(int(n_ws) // 4, 4),), float("nan"), device="cuda") if n_ws else None
    ldb = max(tables.shape[1], -(-max_keys // 16))
    tables = np.pad(tables, ((0, 0), (0, ldb - tables.shape[1])), constant_values=2 ** 30)
    args = (dev(q), dev(pool), len(pool), nq, nkv, hd, len(ns), ints(cu), rows, ints(ctxs), max_q, max_keys, ints(tables), ldb)
    metro.op_attn_tree(*args, out, mask=None if chain else ints(mask), ldm=ldm, workspace=wsp)
    got = host(out)
    again = empty_bits(rows * nq * hd)
    metro.op_attn_tree(*args, again, mask=None if chain else ints(mask), ldm=ldm, workspace=wsp)
    np.testing.assert_array_equal(host(again), got)
    got = bf16_bits_to_f64(got).reshape(rows, nq, hd)
    for i, (c, n) in enumerate(zip(ctxs, ns)):
        k, v = bf16_bits_to_f64(K[i]), bf16_bits_to_f64(V[i])
        see = np.concatenate([np.ones((n, c), bool), seen[i]], axis=1)
        see[:, max_keys:] = False
        ref = D.tree_attention(bf16_bits_to_f64(q[cu[i]:cu[i + 1]]), k, v, see)
        mine = got[cu[i]:cu[i + 1]]
        vm = np.abs(np.where(np.isfinite(v), v, 0.0)).max() if len(v) else 0.0
        with np.errstate(invalid="ignore"):
            bad = ~(np.abs(mine - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -14 + slack) * vm) & ~(np.isnan(mine) & np.isnan(ref)) & (mine != ref)
        assert not bad.any(), (i, c, n, np.argwhere(bad)[:4], mine[bad][:4], ref[bad][:4])
    return got


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_tree(metro, hd, G):
    """Contexts on both sides of pages and page pairs, none at all; trees of one node to three mask words."""
    rng = np.random.default_rng([hd, G])
    tree_case(metro, rng, G, 2, hd, [0, 1, 15, 16, 31, 32, 33, 200], [1, 5, 17, 1, 33, 8, 64, 2])
    tree_case(metro, rng, G, 1, hd, [300, 7], [70, 96], ws=0)
    tree_case(metro, rng, G, 3, hd, [47], [1])


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_chain(metro, hd, G):
    """Without a mask: chunks of a prompt, and single tokens."""
    rng = np.random.default_rng([hd, G, 1])
    tree_case(metro, rng, G, 2, hd, [0, 100, 33], [50, 3, 20], chain=True)
    tree_case(metro, rng, G, 2, hd, [0, 1, 31, 32, 1000], [1] * 5, chain=True)
    tree_case(metro, rng, G, 1, hd, [40], [1], chain=True, ws=0)


@pytest.mark.parametrize("n", [1, 13, 64])
def test_long_contexts_split(metro, n):
    """Splits that end inside and past an item's keys: short items beside long ones, workspaces of every size."""
    rng = np.random.default_rng(n)
    full = metro.op_attn_tree_workspace(8, 2, 128, 3, 3 * n, n, 3500 + n)
    one = 3 * n * 8 * 130 * 4
    for ws in (full, 5 * one + 16, one, 0):
        tree_case(metro, rng, 4, 2, 128, [3500, 5, 1700], [n] * 3, ws=ws)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [1, 8, 20])
def test_long_contexts_without_splits(metro, hd, n):
    """More page pairs a wave than a wave holds page ids of at once (64), on both sides of a multiple of it."""
    rng = np.random.default_rng([hd, n])
    for ctx in (8192 - n, 8192 + 33, 9000):
        tree_case(metro, rng, 4, 1, hd, [ctx], [n], ws=0)


def test_long_chunks_and_wide_trees(metro):
    """Chunks of hundreds of queries in many tiles of columns, masks of many words."""
    rng = np.random.default_rng(21)
    tree_case(metro, rng, 4, 2, 128, [100, 0, 31], [300, 129, 1], chain=True)
    tree_case(metro, rng, 8, 1, 64, [70], [210], chain=True, ws=0)
    tree_case(metro, rng, 2, 2, 128, [45, 200], [200, 31])


def test_bounds_larger_than_any_item(metro):
    """max_q and max_keys of a batch that was planned for more, as a captured one is."""
    rng = np.random.default_rng(22)
    for ws in (True, 0):
        tree_case(metro, rng, 4, 2, 128, [100, 7, 300], [3, 1, 5], max_q=64, max_keys=4096, ws=ws)
        tree_case(metro, rng, 4, 2, 128, [100, 7], [1, 1], chain=True, max_q=3, max_keys=2000, ws=ws)
        tree_case(metro, rng, 1, 3, 64, [100, 7], [9, 2], max_q=30, max_keys=500, ws=ws)


@pytest.mark.parametrize("hd", [64, 128])
def test_many_items(metro, hd):
    """Queries enough that the states are merged a query a workgroup, of one split and of two."""
    rng = np.random.default_rng(5)
    ns = [int(x) for x in rng.integers(1, 12, 60)]
    ctxs = [int(x) for x in rng.integers(0, 300, 60)]
    assert metro.op_attn_tree_workspace(32, 8, hd, 60, sum(ns), max(ns), max(c + n for c, n in zip(ctxs, ns))) > 0
    tree_case(metro, rng, 4, 8, hd, ctxs, ns)


def test_peaked_and_rising_scores(metro):
    rng = np.random.default_rng(6)
    K = [bits(rng.standard_normal((500, 2, 128)) * (0.2 + np.arange(500) / 200)[:, None, None])]
    # (|z| up to 32 * 4: four times the scores' share of the tolerance)
    tree_case(metro, rng, 4, 2, 128, [490], [10], scale=2.0, K=K, slack=2.0 ** -14)
    K = [bits(rng.standard_normal((500, 2, 128)) * (2.7 - np.arange(500) / 200)[:, None, None])]
    tree_case(metro, rng, 4, 2, 128, [490], [10], scale=2.0, K=K, slack=2.0 ** -14)


def test_values_up_to_2_to_the_89(metro):
    """The weights' sums times such values stay within fp32, with scores that rise (a weight may be 2^8 until the maximum that
    it is relative to moves on)."""
    rng = np.random.default_rng(27)
    for hd, G, n, ctx in ((128, 4, 1, 900), (64, 8, 4, 300), (128, 4, 30, 2000)):  # (one tile of columns, two, more)
        rise = (0.2 + 3.0 * np.arange(ctx + n) / (ctx + n))[:, None, None]
        K = [bits(rng.standard_normal((ctx + n, 2, hd)) * rise)]
        V = [bits(np.clip(rng.standard_normal((ctx + n, 2, hd)), -1.99, 1.99) * 2.0 ** 88)]
        for ws in (True, 0):
            # (|z| up to 32 * 4, as above)
            got = tree_case(metro, rng, G, 2, hd, [ctx], [n], scale=2.0, K=K, V=V, ws=ws, slack=2.0 ** -14)
            assert np.isfinite(got).all()


def test_masks_that_leave_rows_empty(metro):
    """No context and no bit: zeros; keys nobody sees hold NaN and Inf."""
    rng = np.random.default_rng(7)
    for hd in (64, 128):
        see = [np.eye(20, dtype=bool), random_tree(rng, 9)]
        see[0][[0, 5, 19]] = False
        K, V = [[bits(rng.standard_normal((n, 2, hd))) for n in (20, 59)] for _ in range(2)]
        for x in (K, V):
            x[0][[0, 5, 19]] = rng.choice(NAN_BITS, size=(3, 2, hd))
        got = tree_case(metro, rng, 4, 2, hd, [0, 50], [20, 9], seen=see, K=K, V=V)
        assert (got[[0, 5, 19]] == 0).all()


def test_masked_values_that_are_not_finite_reach_only_their_queries(metro):
    rng = np.random.default_rng(9)
    for hd in (64, 128):
        K, V = [[bits(rng.standard_normal((48, 2, hd)))] for _ in range(2)]
        V[0][40, :, 3] = 0x7F80
        V[0][41, 1, 5] = 0x7FC0
        V[0][43, 0, hd - 1] = 0xFF80
        K[0][45] = 0x7FC0
        got = tree_case(metro, rng, 2, 2, hd, [38], [10], K=K, V=V)
        assert np.isfinite(got[0]).all() and np.isinf(got[2, :, 3]).all()


def test_infinite_context_values_stay_in_their_outputs(metro):
    """An infinity among the context's values: its dim of its head is infinite or NaN, everything else as without it."""
    rng = np.random.default_rng(25)
    nq, nkv = 16, 2
    for hd, n in ((64, 1), (128, 6), (128, 30)):  # (one tile of columns, three, more)
        K, V = [[bits(rng.standard_normal((200 + n, nkv, hd)))] for _ in range(2)]
        q = bits(rng.standard_normal((n, nq, hd)))

        def go(values):
            pool, tables = tree_pool(np.random.default_rng(26), K, [values], nkv, hd)
            out = empty_bits(n * nq * hd)
            metro.op_attn_tree(dev(q), dev(pool), len(pool), nq, nkv, hd, 1, ints([0, n]), n, ints([200]), n, 200 + n, ints(tables),
                               tables.shape[1], out)
            return bf16_bits_to_f64(host(out)).reshape(n, nkv, nq // nkv, hd)

        plain = go(V[0])
        odd = V[0].copy()
        odd[70, 1, 9] = 0x7F80
        got = go(odd)
        assert np.isfinite(plain).all() and not np.isfinite(got[:, 1, :, 9]).any()
        got[:, 1, :, 9] = plain[:, 1, :, 9]
        assert (got == plain).all()


def test_infinite_scores(metro):
    """Scores of -inf weigh nothing, a query with no others gets zeros."""
    rng = np.random.default_rng(10)
    hd = 64
    K, V = [[bits(np.ones((40, 1, hd))), bits(np.ones((4, 1, hd)))] for _ in range(2)]
    V = [bits(rng.standard_normal(k.shape)) for k in K]
    K[0][7:30] = 0xFF80
    K[1][:] = 0xFF80
    nq = 2
    q = bits(np.full((2, nq, hd), 0.5))
    pool, tables = tree_pool(rng, K, V, 1, hd)
    out = empty_bits(2 * nq * hd)
    metro.op_attn_tree(dev(q), dev(pool), len(pool), nq, 1, hd, 2, ints([0, 1, 2]), 2, ints([39, 3]), 1, 40, ints(tables),
                       tables.shape[1], out)
    got = bf16_bits_to_f64(host(out)).reshape(2, nq, hd)
    v = bf16_bits_to_f64(V[0])[np.r_[0:7, 30:40], 0]
    assert np.all(np.abs(got[0] - v.mean(0)) <= 2.0 ** -8 * np.abs(v.mean(0)) + 2.0 ** -14 * np.abs(v).max())
    assert (got[1] == 0).all()


def test_rows_of_no_item_and_bounds(metro):
    """Rows behind the last item and queries past max_q stay as they were, keys from max_keys on are not seen, and indices
    outside their ranges touch nothing outside the buffers."""
    rng = np.random.default_rng(11)
    hd, nq, nkv = 128, 8, 2
    tree_case(metro, rng, 4, 2, 128, [100, 30], [12, 3], chain=True, max_keys=105)
    K, V = [[bits(rng.standard_normal((60, nkv, hd)))] for _ in range(2)]
    pool, tables = tree_pool(rng, K, V, nkv, hd)
    q = bits(rng.standard_normal((9, nq, hd)))

    def go(cu, ctx, max_q, items, t=tables):
        out = empty_bits(9 * nq * hd)
        metro.op_attn_tree(dev(q), dev(pool), len(pool), nq, nkv, hd, items, ints(cu), 9, ints(ctx), max_q, 60, ints(t),
                           t.shape[1], out)
        return host(out).reshape(9, -1)

    whole = go([2, 7], [50], 5, 1)
    assert (whole[[0, 1, 7, 8]] == 0x7FA5).all() and (whole[2:7] != 0x7FA5).any(axis=1).all()
    part = go([2, 7], [50], 3, 1)
    assert (part[5:] == 0x7FA5).all()
    # (three queries see one another and the 50 keys: the same rows)
    assert np.abs(bf16_bits_to_f64(part[2:5]) - bf16_bits_to_f64(whole[2:5])).max() <= 2.0 ** -7 * np.abs(bf16_bits_to_f64(whole[2:5])).max()
    wild = np.where(tables % 2 == 0, tables, np.int32(2 ** 31 - 1))
    for cu, ctx in (([-5, 100], [2 ** 31 - 1]), ([7, 2], [-3]), ([0, 5], [-2 ** 31])):
        go(cu, ctx, 5, 1, wild)
    both = go([0, 4, 4], [50, 50], 5, 2, np.concatenate([tables, tables]))
    assert (both[4:] == 0x7FA5).all()


def test_cache_past_32_bit_offsets(metro):
    """Pages whose elements lie past 2^32 (8 GiB), and past 2^31 slots' worth of bytes: append, attention and move there."""
    nkv, hd, nq = 8, 128, 8
    page = 2 * nkv * 16 * hd
    n_pages = (1 << 32) // page + 40
    kv = torch.zeros(n_pages * page, dtype=torch.int16, device="cuda")
    rng = np.random.default_rng(12)
    T = 33
    ids = np.array([n_pages - 1, n_pages - 7, n_pages - 3], np.int32)
    slot = ids[np.arange(T) // 16] * 16 + np.arange(T) % 16
    y = rng.standard_normal((T, (nq + 2 * nkv) * hd)).astype(np.float32)
    rope = rope_table(64, hd)
    q = empty_bits(T * nq * hd)
    metro.op_rope_append(dev(y), T, nq, nkv, hd, dev(rope), 64, ints(np.arange(T)), ints(slot), q, kv, n_pages)
    out = empty_bits(T * nq * hd)
    metro.op_attn_tree(q, kv, n_pages, nq, nkv, hd, 1, ints([0, T]), T, ints([0]), T, T, ints(ids), 3, out)
    qr, k, v = D.rope_rows(y, nq, nkv, hd, None, None, 0.0, rope, np.arange(T))
    k, v, qr = [bf16_bits_to_f64(bits(x)) for x in (k, v, qr)]
    ref = D.tree_attention(qr, k, v, np.tril(np.ones((T, T), bool)))
    # (q and k may round to the neighbour: 2^-8 of two factors in scores below 8)
    assert np.abs(bf16_bits_to_f64(host(out)).reshape(T, nq, hd) - ref).max() <= 2.0 ** -5
    metro.op_kv_move(kv, 1, n_pages, nkv, hd, ints([slot[32]]), ints([5]), ints([0, 1]), 1, 1)
    tail = host(kv[-page * 40:]).reshape(40, 2, nkv, 16 * hd)
    head = host(kv[:page]).reshape(2, nkv, 16 * hd)
    for c, places in enumerate(D.tile_places(hd)):
        np.testing.assert_array_equal(head[c][:, places[5]], tail[40 - 3, c][:, places[0]])
    assert (head != 0).sum() <= 2 * nkv * hd
    del kv


# --- kv_move -----------------------------------------------------------------------


@pytest.mark.parametrize("nkv,hd,layers", [(8, 128, 3), (2, 64, 1), (5, 64, 2), (1, 128, 4)])
def test_move(metro, nkv, hd, layers):
    rng = np.random.default_rng([nkv, hd, layers])
    n_pages, gap = 12, 64
    pool = rng.integers(0, 1 << 16, size=(layers, n_pages * 32 * nkv * hd + gap), dtype=np.uint16)
    slots = rng.permutation(n_pages * 16)
    # a path to the front with fixed points, a chain through its own sources, a ring, nothing, slots outside, 40 moves
    src = [[slots[0], slots[3], slots[5]], [slots[11], slots[12], slots[13]], [slots[20], slots[21], slots[22]], [],
           [-1, slots[30], slots[31], 16 * n_pages], list(slots[40:80])]
    dst = [[slots[0], slots[1], slots[2]], [slots[10], slots[11], slots[12]], [slots[21], slots[22], slots[20]], [],
           [slots[32], -5, slots[33], slots[34]], list(slots[90:130])]
    off = np.concatenate([[0], np.cumsum([len(x) for x in src])])
    flat = [np.array([s for x in y for s in x]) for y in (src, dst)]
    kv = dev(pool)
    metro.op_kv_move(kv, layers, n_pages, nkv, hd, ints(flat[0]), ints(flat[1]), ints(off), len(src), len(flat[0]),
                     layer_stride=pool.shape[1])
    body = pool[:, :-gap].reshape(layers, n_pages, 2, nkv, 16 * hd)
    got = host(kv).reshape(layers, -1)
    np.testing.assert_array_equal(got[:, :-gap].reshape(body.shape), D.kv_move(body, hd, flat[0], flat[1], off))
    np.testing.assert_array_equal(got[:, -gap:], pool[:, -gap:])


def test_move_of_long_paths_and_wild_offsets(metro):
    """A compaction of more moves than are read at once; the last of two moves to a slot wins; offsets outside their range."""
    rng = np.random.default_rng(20)
    hd, nkv, n_pages = 64, 2, 10
    pool = rng.integers(0, 1 << 16, size=(1, n_pages, 2, nkv, 16 * hd), dtype=np.uint16)
    src = np.sort(rng.permutation(150)[:90]) + 2
    dst = np.arange(90)
    kv = dev(pool)
    metro.op_kv_move(kv, 1, n_pages, nkv, hd, ints(src), ints(dst), ints([0, 90]), 1, 90)
    np.testing.assert_array_equal(host(kv), D.kv_move(pool, hd, src, dst, [0, 90]))
    kv = dev(pool)
    metro.op_kv_move(kv, 1, n_pages, nkv, hd, ints([9, 70, 11]), ints([1, 1, 2]), ints([0, 3]), 1, 3)
    np.testing.assert_array_equal(host(kv), D.kv_move(pool, hd, [9, 70, 11], [1, 1, 2], [0, 3]))
    kv = dev(pool)
    metro.op_kv_move(kv, 1, n_pages, nkv, hd, ints([9, 70, 11]), ints([1, 3, 2]), ints([-4, 1, 2 ** 31 - 1]), 2, 3)
    np.testing.assert_array_equal(host(kv), D.kv_move(pool, hd, [9, 70, 11], [1, 3, 2], [0, 3]))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n", [9, 16, 17, 40])
def test_move_of_paths_over_pages_in_any_order(metro, hd, n):
    """Accepted paths of more moves than are read at once, to places among their own sources, over pages whose ids fall or
    have no order: as if all sources were read first."""
    rng = np.random.default_rng([hd, n])
    nkv, n_pages = 2, 24
    for ids in (np.arange(n_pages)[::-1], rng.permutation(n_pages)):
        for layers, first in ((1, 0), (2, 13)):
            pool = rng.integers(0, 1 << 16, size=(layers, n_pages, 2, nkv, 16 * hd), dtype=np.uint16)
            src, dst, off = [], [], [0]
            for seq in range(3):
                at = lambda o: ids[8 * seq + o // 16] * 16 + o % 16
                # the root, then nodes at or behind the path's own places, close to them
                nodes = first + np.arange(n) + np.concatenate([[0], np.sort(rng.integers(0, 20 + 3 * seq, n - 1))])
                src += [int(at(o)) for o in nodes]
                dst += [int(at(first + j)) for j in range(n)]
                off.append(len(src))
            kv = dev(pool)
            metro.op_kv_move(kv, layers, n_pages, nkv, hd, ints(src), ints(dst), ints(off), 3, len(src))
            np.testing.assert_array_equal(host(kv), D.kv_move(pool, hd, src, dst, off))


def test_long_exchanges_go_eight_at_a_time(metro):
    rng = np.random.default_rng(42)
    hd, nkv, n_pages = 64, 2, 10
    pool = rng.integers(0, 1 << 16, size=(1, n_pages, 2, nkv, 16 * hd), dtype=np.uint16)
    slots = rng.permutation(n_pages * 16)[:30]
    src, dst = slots, np.roll(slots, -1)
    want = pool
    for lo in range(0, 30, 8):
        want = D.kv_move(want, hd, src[lo:lo + 8], dst[lo:lo + 8], [0, len(src[lo:lo + 8])])
    kv = dev(pool)
    metro.op_kv_move(kv, 1, n_pages, nkv, hd, ints(src), ints(dst), ints([0, 30]), 1, 30)
    np.testing.assert_array_equal(host(kv), want)


# --- sample --------------------------------------------------------------------------


def sample_case(metro, x, u, ldl=None, **settings):
    """Rows x [rows, vocab] with settings as lists (None: not given); compares with the definition and returns the tokens."""
    x = np.asarray(x, np.float32)
    rows, vocab = x.shape
    ldl = ldl or vocab
    full = np.full((rows, ldl), np.inf, np.float32)  # (what lies behind the vocabulary says nothing)
    full[:, :vocab] = x
    arrays = {k: None if v is None else np.asarray(v, np.int32 if k == "top_k" else np.float32) for k, v in settings.items()}
    u = np.asarray(u, np.float32)
    out, prob = ints(np.full(rows, -9)), torch.full((rows,), -1.0, device="cuda")
    n = metro.op_sample_workspace(rows, vocab)
    ws = torch.full((max(n, 16),), 0xA5, dtype=torch.uint8, device="cuda")
    given = {k: None if v is None else dev(v) for k, v in arrays.items()}
    for _ in range(2):  # (the second call finds what the first left in the workspace)
        metro.op_sample(dev(full), rows, vocab, dev(u), out, prob=prob, ldl=ldl, workspace=ws, **given)
        tokens, probs = host(out).copy(), host(prob).astype(np.float64)
        for r in range(rows):
            t, p = D.sample(x[r], float(u[r]), **{k: v[r].item() for k, v in arrays.items() if v is not None})
            assert tokens[r] == t, (r, tokens[r], t, {k: v[r].item() for k, v in arrays.items() if v is not None}, float(u[r]))
            assert abs(probs[r] - p) <= 2.0 ** -24 * p + 2.0 ** -28, (r, probs[r], p)
        out.fill_(-9)
    return tokens


def logits(rng, rows, vocab, spread=2.0):
    x = spread * rng.standard_normal((rows, vocab))
    for r in range(rows):
        at = rng.integers(0, vocab, 12)
        x[r, at] += 10 * rng.random(12)
    return x.astype(np.float32)


VOCABS = [1, 2, 5, 63, 1000, 1025, 4096, 4099, 32000, 50257, 128256, 262144]


@pytest.mark.parametrize("vocab", VOCABS)
def test_sample_settings(metro, vocab):
    rng = np.random.default_rng(vocab)
    rows = 24 if vocab < 50000 else 8
    x = logits(rng, rows, vocab)
    pick = lambda *v: rng.choice(v, rows)
    for kw in (dict(), dict(temperature=pick(0.3, 0.7, 1.0, 2.5)), dict(top_k=pick(1, 2, 50, 1000, 10 ** 9)),
               dict(top_p=pick(0.1, 0.5, 0.9, 0.99)), dict(min_p=pick(0.01, 0.1, 0.5, 1.0)),
               dict(temperature=pick(0.0, 0.8, 1.3), top_k=pick(0, 40, 500), top_p=pick(1.0, 0.95, 0.6), min_p=pick(0.0, 0.02))):
        sample_case(metro, x, rng.random(rows), ldl=vocab + int(rng.integers(0, 3)), **kw)


def test_sample_bounds_of_u(metro):
    rng = np.random.default_rng(1)
    x = np.repeat(logits(rng, 1, 5000), 8, axis=0)
    u = [0.0, np.float32(1) - np.float32(2.0 ** -24), 1.0, 5.0, -1.0, np.nan, np.inf, -np.inf]
    for kw in (dict(), dict(top_k=[7] * 8), dict(top_p=[0.8] * 8), dict(min_p=[0.05] * 8)):
        tokens = sample_case(metro, x, u, **kw)
        assert tokens[0] == tokens[4] == tokens[5] == tokens[7] == int(np.argmax(x[0])) and tokens[2] == tokens[3] == tokens[6]


def clear_border(x, temperature):
    """Rows without weights between 2^-46.3 and 2^-45.9, which may or may not count as none."""
    t = np.asarray(temperature, np.float64).reshape(-1, 1)
    bits_below = (x.max(axis=1, keepdims=True).astype(np.float64) - x) / t / np.log(2.0)
    x = np.where((bits_below > 45.9) & (bits_below < 46.3), x - (0.5 * t).astype(np.float32), x).astype(np.float32)
    bits_below = (x.max(axis=1, keepdims=True).astype(np.float64) - x) / t / np.log(2.0)
    assert not ((bits_below > 45.9) & (bits_below < 46.3)).any()
    return x


@pytest.mark.parametrize("vocab", [777, 5000])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 1.7])
def test_sample_last_kept_token(metro, vocab, temperature):
    """u from 1 on gives the last kept token: rows in many of which the bin of min-p's least weight holds tokens and keeps
    none, so that the sum that is left and the last token's own are rounded apart."""
    rng = np.random.default_rng([vocab, int(10 * temperature)])
    rows = 240
    x = clear_border((2.0 * rng.standard_normal((rows, vocab))).astype(np.float32), np.full(rows, temperature))
    u = rng.choice([1.0, 5.0, np.inf], rows)
    pick = lambda *v: rng.choice(v, rows)
    t = np.full(rows, temperature)
    for kw in (dict(), dict(min_p=pick(0.001, 0.02, 0.05, 0.1)), dict(min_p=pick(0.001, 0.05), top_k=pick(3, 40, 300, 10 ** 6)),
               dict(min_p=pick(0.001, 0.05), top_p=pick(0.3, 0.9, 0.999)), dict(top_k=pick(1, 60, 700), top_p=pick(0.2, 0.95)),
               dict(min_p=pick(0.0, 0.01), top_k=pick(0, 20, 500), top_p=pick(1.0, 0.99))):
        sample_case(metro, x, u, temperature=t, **kw)


def test_sample_last_kept_token_of_light_tails(metro):
    """Weights that the running sums lose, alone in their bin, crowded in it, and equal."""
    rng = np.random.default_rng(41)
    vocab = 200000
    one = np.zeros(vocab, np.float32)
    one[777] = -31.0
    some = np.zeros(vocab, np.float32)
    some[rng.permutation(vocab)[:300]] = (-31.0 - 0.01 * rng.random(300)).astype(np.float32)
    same = np.zeros(vocab, np.float32)
    same[rng.permutation(vocab)[:5000]] = -30.5
    none = np.zeros(vocab, np.float32)
    none[5] = -40.0  # (below 2^-46: as good as not there)
    x = np.stack([one, some, same, none] * 3)
    u = np.repeat([1.0, 7.0, np.inf], 4)
    sample_case(metro, x, u)
    sample_case(metro, x, u, top_k=[vocab - 1, vocab - 150, vocab - 2500, vocab - 1] * 3)
    sample_case(metro, x, u, min_p=[0.5, 3.425e-14, 5e-14, 1e-13] * 3)  # (none of one's, some of some's, all of same's)
    sample_case(metro, x, u, top_p=[0.9] * 12)


@pytest.mark.parametrize("vocab", [300, 5000, 20000])
def test_sample_last_kept_token_of_odd_rows(metro, vocab):
    """Ties, signed zeros, crowded logits, infinities, NaN and one token alone, with u from 1 on."""
    rng = np.random.default_rng([vocab, 43])
    nan, inf = np.nan, np.inf
    some = lambda share, a, b: np.where(rng.random(vocab) < share, np.float32(a), b)
    steps = (-np.arange(vocab) // 300 / 8).astype(np.float32)
    rng.shuffle(steps)
    x = np.stack([np.full(vocab, 1.5), some(0.5, 2.0, 1.0), some(0.5, 0.0, -0.0), steps, 8.0 + 1e-3 * rng.random(vocab),
                  1e-30 * rng.standard_normal(vocab), some(0.1, 3.0, -1e4 * rng.random(vocab)),
                  1e6 + 64 * rng.integers(0, 3, vocab), some(0.7, -inf, rng.standard_normal(vocab)),
                  some(0.7, nan, rng.standard_normal(vocab)), some(0.01, inf, rng.standard_normal(vocab)),
                  np.where(np.arange(vocab) == 7, 2.0, nan), np.full(vocab, -inf)]).astype(np.float32)
    x[:8] = clear_border(x[:8], np.ones(8))
    rows = len(x)
    u = rng.choice([1.0, 3.0, inf], rows)
    pick = lambda *v: rng.choice(v, rows)
    for kw in (dict(), dict(top_k=pick(1, 2, 100, 290, 10 ** 9)), dict(top_p=pick(0.05, 0.31, 0.9)), dict(min_p=pick(0.01, 0.5, 1.0)),
               dict(min_p=pick(0.01, 0.9), top_k=pick(0, 97, 280), top_p=pick(1.0, 0.55, 0.99)), dict(temperature=np.zeros(rows))):
        tokens = sample_case(metro, x, u, **kw)
        assert tokens[11] == 7 and tokens[12] == -1


def test_sample_odd_settings(metro):
    rng = np.random.default_rng(2)
    x = logits(rng, 8, 3001)
    u = rng.random(8)
    nan, inf = np.nan, np.inf
    sample_case(metro, x, u, temperature=[nan, -1.0, 0.0, inf, 1e-30, 1e-45, 1e30, 0.01])
    sample_case(metro, x, u, top_p=[nan, -1.0, 0.0, inf, 1.0, 1e-30, 1.5, -inf], top_k=[0, -5, 1, 3001, 3002, 2 ** 31 - 1, -2 ** 31, 2])
    sample_case(metro, x, u, min_p=[nan, -1.0, 0.0, inf, 1.0, 1e-30, 1.5, -inf], top_p=[0.9] * 8)


@pytest.mark.parametrize("vocab", [300, 5000, 128256])
def test_sample_ties(metro, vocab):
    """Equal logits, in all tokens or in many of them, signed zeros: the order goes by the index."""
    rng = np.random.default_rng(vocab)
    flat = np.full(vocab, 1.5, np.float32)
    two = np.where(rng.random(vocab) < 0.5, np.float32(2.0), np.float32(1.0))
    zeros = np.where(rng.random(vocab) < 0.5, np.float32(0.0), np.float32(-0.0))
    steps = (-np.arange(vocab) // 300 / 8).astype(np.float32)
    rng.shuffle(steps)
    x = np.stack([flat, two, zeros, steps] * 2)
    u = rng.random(8)
    for kw in (dict(), dict(top_k=[2, 280, 50, 290, 299, 100, 1, 3]), dict(top_p=[0.3, 0.61, 0.77, 0.5, 0.9, 0.1, 0.2, 0.4]),
               dict(top_k=[100] * 8, top_p=[0.55] * 8, temperature=[0.7] * 8), dict(min_p=[1.0] * 8)):
        sample_case(metro, x, u, **kw)


def test_sample_crowded_logits(metro):
    """Thousands of different logits within a small step of one another, and next to zero."""
    rng = np.random.default_rng(3)
    x = np.stack([8.0 + 1e-3 * rng.random(20000), 1e-3 * rng.standard_normal(20000), 1e-30 * rng.standard_normal(20000),
                  np.where(rng.random(20000) < 0.1, 3.0, -1e4 * rng.random(20000)), 1e6 + 64 * rng.integers(0, 3, 20000),
                  1e-42 * rng.standard_normal(20000)]).astype(np.float32)
    for kw in (dict(), dict(top_k=[300, 1500, 5000, 1999, 700, 9999]), dict(top_p=[0.5, 0.31, 0.77, 0.9, 0.2, 0.6]),
               dict(temperature=[1e-3, 1e-3, 1e-30, 1.0, 100.0, 1e-42], top_p=[0.8] * 6)):
        sample_case(metro, x, rng.random(6), **kw)


@pytest.mark.parametrize("spread", [0.01, 1.0, 20.0])
def test_sample_many_rows_of_many_settings(metro, spread):
    rng = np.random.default_rng(int(100 * spread))
    rows, vocab = 1500, 777
    x = (spread * rng.standard_normal((rows, vocab))).astype(np.float32)
    x[::3] = np.round(x[::3] * 4 / spread) * (spread / 4)  # (ties)
    pick = lambda *v: rng.choice(v, rows)
    sample_case(metro, x, rng.random(rows), temperature=pick(0.0, 0.2, 0.7, 1.0, 3.0), top_k=pick(0, 1, 5, 30, 300, 776),
                top_p=pick(0.05, 0.5, 0.9, 0.999, 1.0), min_p=pick(0.0, 0.0, 0.01, 0.3, 0.9))


def test_sample_infinities_and_nan(metro):
    rng = np.random.default_rng(4)
    x = logits(rng, 9, 2000)
    nan, inf = np.nan, np.inf
    x[0] = -inf
    x[1] = nan
    x[2, :-1] = nan
    x[3, 1:] = -inf
    x[4, rng.permutation(2000)[:1500]] = -inf
    x[5, rng.permutation(2000)[:1500]] = nan
    x[6, [7, 700]] = inf
    x[7, 5] = inf
    x[8, :] = np.where(rng.random(2000) < 0.5, nan, -inf)
    u = rng.random(9)
    for kw in (dict(), dict(top_k=[3] * 9), dict(top_p=[0.7] * 9), dict(min_p=[0.1] * 9), dict(temperature=[0.0] * 9)):
        tokens = sample_case(metro, x, u, **kw)
        assert list(tokens[[0, 1, 8]]) == [-1] * 3 and tokens[2] == 1999 and tokens[3] == 0 and tokens[7] == 5


def test_sample_follows_the_distribution(metro):
    """20000 draws from one row: counts within six standard deviations of their expectation."""
    rng = np.random.default_rng(5)
    x = np.log([0.4, 0.05, 0.3, 0.25]).astype(np.float32)
    n = 20000
    out = ints(np.zeros(n))
    ws = torch.empty(max(metro.op_sample_workspace(n, 4), 16), dtype=torch.uint8, device="cuda")
    metro.op_sample(dev(np.repeat(x[None], n, axis=0)), n, 4, dev(rng.random(n).astype(np.float32)), out, workspace=ws)
    counts = np.bincount(host(out), minlength=4)
    p = np.exp(x.astype(np.float64))
    assert np.all(np.abs(counts - n * p) <= 6 * np.sqrt(n * p * (1 - p)))


# --- nothing outside the buffers -----------------------------------------------------

GUARD = 1 << 16  # bytes before and behind a buffer
INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


class Guarded:
    """A device buffer between guards of a known pattern."""

    def __init__(self, content):
        raw = np.ascontiguousarray(content).view(np.uint8).ravel()
        self.n = raw.size
        self.was = np.random.default_rng(77).integers(0, 256, 2 * GUARD, dtype=np.uint8)
        self.all = dev(np.concatenate([self.was[:GUARD], raw, self.was[GUARD:]]))
        self.inner = self.all[GUARD:GUARD + self.n]

    def read(self, dtype):
        """The buffer's content, once its guards are as they were."""
        a = host(self.all)
        np.testing.assert_array_equal(a[:GUARD], self.was[:GUARD])
        np.testing.assert_array_equal(a[GUARD + self.n:], self.was[GUARD:])
        return a[GUARD:GUARD + self.n].view(dtype)


@pytest.mark.parametrize("hd", [64, 128])
def test_append_touches_nothing_outside(metro, hd):
    """Slots on both sides of the cache's ends, in runs and alone; positions outside the table."""
    rng = np.random.default_rng([hd, 50])
    nq, nkv, n_pages, end = 4, 2, 3, 48
    slot = np.array([end - 2, end - 1, end, end + 1, end, end + 1, end + 2, end + 3, -4, -3, -2, -1, -1, 0, 1, 2, 3, 20, INT_MIN,
                     INT_MAX, INT_MAX - 3, INT_MAX - 2, INT_MAX - 1, end + 16, 44], np.int64)
    pos = rng.integers(0, 30, len(slot))
    pos[[1, 4, 17]] = INT_MIN, INT_MAX, -1
    T, width = len(slot), (nq + 2 * nkv) * hd
    y = rng.standard_normal((T, width)).astype(np.float32)
    rope = rope_table(30, hd)
    pool = rng.choice(NAN_BITS, size=(n_pages, 2, nkv, 16 * hd))
    for rows in (dev(y), dev(bits(y)).view(torch.bfloat16)):
        kv, q = Guarded(pool), Guarded(np.full(T * nq * hd, 0x7FA5, np.uint16))
        metro.op_rope_append(rows, T, nq, nkv, hd, dev(rope), 30, ints(pos), ints(slot), q.inner, kv.inner, n_pages)
        turned = bf16_bits_to_f64(q.read(np.uint16)).reshape(T, -1)
        np.testing.assert_array_equal(np.isnan(turned).all(axis=1), (pos < 0) | (pos >= 30))
        got, left, places = kv.read(np.uint16).reshape(pool.shape), pool.copy(), D.tile_places(hd)
        for s in slot[(slot >= 0) & (slot < end)]:
            for c in range(2):
                at = places[c][s % 16]
                assert not np.isin(got[s // 16, c][:, at], NAN_BITS[2:]).any()
                left[s // 16, c][:, at] = got[s // 16, c][:, at]
        np.testing.assert_array_equal(got, left)


@pytest.mark.parametrize("hd,G,n", [(64, 1, 5), (128, 4, 1), (128, 4, 7), (64, 8, 9), (128, 2, 40)])
def test_tree_touches_nothing_outside(metro, hd, G, n):
    """Workspaces of just the queried size and of less, row ranges, contexts and pages outside theirs: the rows that an item
    has are written, and no others."""
    rng = np.random.default_rng([hd, G, n])
    nkv, rows, max_keys = 2, 2 * n + 3, 1500
    nq, pages = G * nkv, 20
    pool = bits(rng.standard_normal((pages, 2, nkv, 16 * hd)))
    q = bits(rng.standard_normal((rows, nq, hd)))
    kv, qd = dev(pool), dev(q)
    ldb = -(-max_keys // 16)
    wild = rng.choice(np.array([INT_MIN, -1, 0, 5, pages - 1, pages, INT_MAX], np.int64), size=(2, ldb))
    need = metro.op_attn_tree_workspace(nq, nkv, hd, 2, rows, n, max_keys)
    state = rows * nq * (hd + 2) * 4
    assert need > 2 * state
    cases = [([1, 1 + n, 1 + 2 * n], [1500 - n, 33]), ([-5, n, INT_MAX], [INT_MAX, INT_MIN]), ([INT_MIN, 0, rows], [7, 1400]),
             ([rows, INT_MAX, INT_MAX], [1, 1]), ([n, 2, 2], [-9, 40])]
    for size in (need, need - 4, 2 * state, 2 * state - 4, 0):
        for cu, ctx in cases:
            ws, out = Guarded(np.full(max(size, 4), 0xA5, np.uint8)), Guarded(np.full(rows * nq * hd, 0x7FA5, np.uint16))
            metro.op_attn_tree(qd, kv, pages, nq, nkv, hd, 2, ints(cu), rows, ints(ctx), n, max_keys, ints(wild), ldb, out.inner,
                               workspace=ws.inner.view(torch.float32) if size else None)
            ws.read(np.uint8)
            got = out.read(np.uint16).reshape(rows, -1)
            mine = np.zeros(rows, bool)
            for i in range(2):
                lo = min(max(cu[i], 0), rows)
                mine[lo:max(lo, min(min(max(cu[i + 1], 0), rows), lo + n))] = True
            np.testing.assert_array_equal((got != 0x7FA5).any(axis=1), mine)
            np.testing.assert_array_equal((got != 0x7FA5).all(axis=1), mine)


def test_move_touches_nothing_outside(metro):
    rng = np.random.default_rng(51)
    nkv, hd, n_pages, end = 3, 64, 4, 64
    pool = rng.integers(0, 1 << 16, size=(2, n_pages, 2, nkv, 16 * hd), dtype=np.uint16)
    src = np.array([end, end - 1, -1, 5, 6, INT_MIN, INT_MAX, 7, 8, 9, end + 15], np.int64)
    dst = np.array([1, end, 2, 10, INT_MAX, 3, 4, INT_MIN, end + 1, 0, end + 31], np.int64)
    kv = Guarded(pool)
    metro.op_kv_move(kv.inner, 2, n_pages, nkv, hd, ints(src), ints(dst), ints([INT_MIN, 4, INT_MAX]), 2, len(src))
    np.testing.assert_array_equal(kv.read(np.uint16).reshape(pool.shape), D.kv_move(pool, hd, src, dst, [0, 4, len(src)]))


@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 777), (5, 16385), (2, 128256)])
def test_sample_touches_nothing_outside(metro, rows, vocab):
    rng = np.random.default_rng([rows, vocab])
    x = logits(rng, rows, vocab)
    ws = Guarded(np.full(metro.op_sample_workspace(rows, vocab), 0xA5, np.uint8))
    u = rng.random(rows).astype(np.float32)
    for top_k in (0, 30, INT_MAX):
        out, prob = Guarded(np.full(rows, -9, np.int32)), Guarded(np.full(rows, -1, np.float32))
        metro.op_sample(dev(x), rows, vocab, dev(u), out.inner, top_k=ints([top_k] * rows), prob=prob.inner, workspace=ws.inner)
        ws.read(np.uint8)
        tokens, probs = out.read(np.int32), prob.read(np.float32)
        for r in range(rows):
            t, p = D.sample(x[r], float(u[r]), top_k=top_k)
            assert tokens[r] == t and abs(float(probs[r]) - p) <= 2.0 ** -24 * p + 2.0 ** -28


# --- together ------------------------------------------------------------------------


def build(rng, layers, nq, nkv, hd, n_pages):
    return dict(layers=layers, nq=nq, nkv=nkv, hd=hd, n_pages=n_pages, rope=dev(rope_table(600, hd)),
                gains=[dev(bits(1 + 0.1 * rng.standard_normal(hd))) for _ in range(2)])


def append(metro, m, kv, y, pos, slot):
    q = empty_bits(len(pos) * m["nq"] * m["hd"])
    metro.op_rope_append(dev(y), len(pos), m["nq"], m["nkv"], m["hd"], m["rope"], 600, ints(pos), ints(slot), q, kv, m["n_pages"],
                         q_gain=m["gains"][0], k_gain=m["gains"][1], eps=EPS)
    return q


def test_speculative_step_equals_the_plain_one(metro):
    """Two sequences, trees of drafts appended behind their contexts, attended to, an accepted path moved to the front: the
    cache then holds, bit for bit, what appending the accepted tokens one after another puts there, attention over the
    accepted nodes gave what single queries over that cache give, and metro_op_attn_decode agrees."""
    rng = np.random.default_rng(30)
    layers, nq, nkv, hd, n_pages = 2, 8, 2, 128, 40
    m = build(rng, layers, nq, nkv, hd, n_pages)
    width = (nq + 2 * nkv) * hd
    ctxs, n = [77, 300], 12
    parents = [-1, 0, 0, 1, 1, 2, 3, 4, 4, 6, 8, 8]
    see = np.eye(n, dtype=bool)
    depth = np.zeros(n, int)
    for r in range(1, n):
        see[r] |= see[parents[r]]
        depth[r] = depth[parents[r]] + 1
    path = [0, 1, 4, 8, 11]
    ids = rng.permutation(n_pages)
    need = [-(-(c + n) // 16) for c in ctxs]
    tables = np.zeros((2, max(need)), np.int32)
    tables[0, :need[0]], tables[1, :need[1]] = ids[:need[0]], ids[need[0]:sum(need)]
    at = lambda i, o: tables[i][np.asarray(o) // 16] * 16 + np.asarray(o) % 16
    kv = torch.zeros((layers, n_pages * 32 * nkv * hd), dtype=torch.int16, device="cuda")
    plain = torch.zeros_like(kv)
    mask, ldm = pack_mask([see, see], n)
    ws = torch.empty(max(metro.op_attn_tree_workspace(nq, nkv, hd, 2, 2 * n, n, 312) // 4, 4), device="cuda")
    drafted, single = [], []
    for layer in range(layers):
        ctx_rows = [rng.standard_normal((c, width)).astype(np.float32) for c in ctxs]
        draft_rows = [rng.standard_normal((n, width)).astype(np.float32) for _ in ctxs]
        for where in (kv, plain):
            for i, c in enumerate(ctxs):
                append(metro, m, where[layer], ctx_rows[i], np.arange(c), at(i, np.arange(c)))
        q = append(metro, m, kv[layer], np.concatenate(draft_rows), np.concatenate([c + depth for c in ctxs]),
                   np.concatenate([at(i, c + np.arange(n)) for i, c in enumerate(ctxs)]))
        out = empty_bits(2 * n * nq * hd)
        metro.op_attn_tree(q, kv[layer], n_pages, nq, nkv, hd, 2, ints([0, n, 2 * n]), 2 * n, ints(ctxs), n, 312, ints(tables),
                           tables.shape[1], out, mask=ints(mask), ldm=ldm, workspace=ws)
        drafted.append(bf16_bits_to_f64(host(out)).reshape(2, n, nq * hd)[:, path])
        steps = []
        for d, node in enumerate(path):
            y = np.stack([draft_rows[i][node] for i in range(2)])
            q = append(metro, m, plain[layer], y, np.array(ctxs) + d, [int(at(i, c + d)) for i, c in enumerate(ctxs)])
            out = empty_bits(2 * nq * hd)
            metro.op_attn_tree(q, plain[layer], n_pages, nq, nkv, hd, 2, ints([0, 1, 2]), 2, ints(np.array(ctxs) + d), 1, 312,
                               ints(tables), tables.shape[1], out, workspace=ws)
            known = empty_bits(2 * nq * hd)
            ctx = np.array(ctxs) + d + 1
            metro.op_attn_decode(q, plain[layer], n_pages, nq, nkv, hd, ctx,
                                 np.concatenate([tables[i, :-(-int(c) // 16)] for i, c in enumerate(ctx)]), known)
            a, b = bf16_bits_to_f64(host(out)), bf16_bits_to_f64(host(known))
            # (each within half a bf16 step and 2^-14 max |v| of the same value)
            assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.maximum(np.abs(a), np.abs(b)) + 2.0 ** -13 * 5)
            steps.append(a.reshape(2, nq * hd))
        single.append(np.stack(steps, axis=1))
    src = np.concatenate([at(i, np.array(path) + c) for i, c in enumerate(ctxs)])
    dst = np.concatenate([at(i, np.arange(len(path)) + c) for i, c in enumerate(ctxs)])
    metro.op_kv_move(kv, layers, n_pages, nkv, hd, ints(src), ints(dst), ints([0, len(path), 2 * len(path)]), 2, len(src))
    a, b = [host(x).reshape(layers, n_pages, 2, nkv, 16 * hd) for x in (kv, plain)]
    for c, places in enumerate(D.tile_places(hd)):
        for i, ctx in enumerate(ctxs):
            for t in at(i, np.arange(ctx + len(path))):
                np.testing.assert_array_equal(a[:, t // 16, c][..., places[t % 16]], b[:, t // 16, c][..., places[t % 16]])
    for x, y in zip(drafted, single):
        assert np.all(np.abs(x - y) <= 2.0 ** -7 * np.maximum(np.abs(x), np.abs(y)) + 2.0 ** -13 * 5)


def test_captured_step_replays(metro):
    """The run of operators captured into a graph and replayed with new contents of its buffers, eager work and
    synchronizations between: every replay equals the eager run.  Two graphs with workspaces of their own alternate."""
    rng = np.random.default_rng(31)
    nq, nkv, hd, n_pages, T, vocab = 8, 2, 128, 64, 14, 5003
    m = build(rng, 1, nq, nkv, hd, n_pages)
    width = (nq + 2 * nkv) * hd

    def state(salt):
        r = np.random.default_rng(salt)
        return dict(y=dev(r.standard_normal((T, width)).astype(np.float32)), pos=ints(np.arange(T) % 7 + 400),
                    slot=ints(np.concatenate([np.arange(7) + 400, 16 * 32 + np.arange(7) + 400])), q=empty_bits(T * nq * hd),
                    kv=dev(bits(r.standard_normal((n_pages, 32 * nkv * hd)))), out=empty_bits(T * nq * hd),
                    ctx=ints([400, 400]), cu=ints([0, 7, 14]), tables=ints(np.arange(64).reshape(2, 32)),
                    x=dev(logits(r, T, vocab)), u=dev(r.random(T).astype(np.float32)), token=ints(np.zeros(T)),
                    prob=torch.zeros(T, device="cuda"), top_p=dev(np.full(T, 0.9, np.float32)),
                    top_k=ints([0, 40] * 7), src=ints([402, 405, 16 * 32 + 401]), dst=ints([401, 402, 16 * 32 + 400]),
                    off=ints([0, 2, 3]),
                    ws=torch.empty(max(metro.op_attn_tree_workspace(nq, nkv, hd, 2, T, 7, 407) // 4, 4), device="cuda"),
                    ws2=torch.empty(max(metro.op_sample_workspace(T, vocab), 16), dtype=torch.uint8, device="cuda"))

    def step(s):
        metro.op_rope_append(s["y"], T, nq, nkv, hd, m["rope"], 600, s["pos"], s["slot"], s["q"], s["kv"], n_pages,
                             q_gain=m["gains"][0], k_gain=m["gains"][1])
        metro.op_attn_tree(s["q"], s["kv"], n_pages, nq, nkv, hd, 2, s["cu"], T, s["ctx"], 7, 407, s["tables"], 32, s["out"],
                           workspace=s["ws"])
        metro.op_sample(s["x"], T, vocab, s["u"], s["token"], top_k=s["top_k"], top_p=s["top_p"], prob=s["prob"], workspace=s["ws2"])
        metro.op_kv_move(s["kv"], 1, n_pages, nkv, hd, s["src"], s["dst"], s["off"], 2, 3)

    outputs = ("q", "kv", "out", "token", "prob")
    states, graphs = [state(1), state(2)], []
    for s in states:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(s)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(s)
        graphs.append(g)
    for turn in range(4):
        fresh = [state(10 + 2 * turn + i) for i in range(2)]
        eager = [state(10 + 2 * turn + i) for i in range(2)]
        for e in eager:
            step(e)
        for s, f in zip(states, fresh):
            for k in s:
                if k not in ("ws", "ws2"):
                    s[k].copy_(f[k])
        order = (0, 1) if turn % 2 else (1, 0)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for s, e in zip(states, eager):
            for k in outputs:
                np.testing.assert_array_equal(host(s[k]), host(e[k]), err_msg=f"{turn} {k}")


def test_calls_on_two_streams_at_once(metro):
    rng = np.random.default_rng(32)
    rows, vocab = 40, 30011
    x, u = dev(logits(rng, rows, vocab)), dev(rng.random(rows).astype(np.float32))
    top_p = dev(np.full(rows, 0.95, np.float32))
    torch.cuda.synchronize()
    outs = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams + [None]:
        out = ints(np.zeros(rows))
        ws = torch.empty(max(metro.op_sample_workspace(rows, vocab), 16), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize() if s is None else s.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            metro.op_sample(x, rows, vocab, u, out, top_p=top_p, workspace=ws, stream=s)
        outs.append((out, ws))
    torch.cuda.synchronize()
    for out, _ in outs[1:]:
        np.testing.assert_array_equal(host(out), host(outs[0][0]))
