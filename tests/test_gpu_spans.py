"""Windows with sinks and trees of drafted tokens on the GPU, against their definitions in 64 bits (tolerance: spans_reference.within)."""
import numpy as np
import pytest
import torch

from e4m3_reference import held
from paper_2501_05408_amd import synth
from paper_2501_05408_amd import tempo as T
from paper_2501_05408_amd.store import BlockStore
from spans_reference import ancestors, attention, depths, sees_chain, sees_tree, turned, within, within_fp32

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
STORES = [T.TEMPO_BF16, T.TEMPO_E4M3]
ALL_STORES = STORES + [T.TEMPO_F32]
UNTOUCHED = 7.0


def np64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV).to(torch.bfloat16)


def rows_of(dtype, x):
    return bf16(x) if dtype != T.TEMPO_F32 else torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DEV)


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def normal(seed, which, shape, dtype=T.TEMPO_BF16):
    return synth.normal_as(seed, which, shape, "f32" if dtype == T.TEMPO_F32 else "bf16").astype(np.float64)


def near(dtype, got, q, K, V, seen):
    out, size = attention(q, kept(dtype, K), kept(dtype, V), seen)
    within_fp32(got, out, size, q, K) if dtype == T.TEMPO_F32 else within(got, out, size)


def make_store(seed, dtype, B, Hq, Hkv, D, Z, max_t):
    """Blocks in a random order, NaN wherever nothing is written."""
    columns = max_t // Z + 1
    n = B * columns + 3
    table = torch.from_numpy(synth.permutation(seed, 77, n)[:B * columns].reshape(B, columns).copy())
    return BlockStore(B, Hq, Hkv, D, Z, max_t, dtype, device=DEV, num_blocks=n, block_table=table, fill="nan")


def kept(dtype, x):
    return held(x) if dtype == T.TEMPO_E4M3 else x


def write_lengths(st, K, V, lengths):
    """Steps 0 .. lengths[b]-1 of each sequence."""
    for n in sorted(set(int(x) for x in lengths)):
        if n == 0:
            continue
        some = [b for b in range(st.batch) if lengths[b] == n]
        kv = T.make_kv(st.k_pool, st.v_pool, st.block_table[some].contiguous(), st.num_blocks, st.max_blocks_per_seq, st.Z, st.Hkv, st.D, st.dtype)
        keep = st.block_table[some].contiguous()
        kv.block_table = keep.data_ptr()
        T.tempo_kv_append_block(kv, rows_of(st.dtype, K[some, :n]), rows_of(st.dtype, V[some, :n]), len(some), 0, None, n)
        torch.cuda.synchronize()


def tree_of(kind, n, rng):
    if kind == "chain":
        return np.arange(n) - 1
    if kind == "star":
        return np.full(n, -1)
    p = np.array([rng.integers(-1, i) if i else -1 for i in range(n)])
    if kind == "deep":
        p = np.array([max(-1, i - 1 - int(rng.integers(0, 3))) for i in range(n)])
    return p


def pick_steps(rng, t, B, ragged):
    steps = np.full(B, t)
    if ragged:
        steps = np.array([t] + [int(rng.integers(0, t + 1)) for _ in range(B - 1)])[:B]
    return steps


TREES = [  # Hq, Hkv, D, Z, B, t, nodes, kind, window, sinks, ragged, counts
    (24, 8, 128, 64, 2, 300, 8, "random", 0, 0, False, False),
    (6, 2, 128, 32, 3, 0, 5, "random", 0, 0, False, False),
    (4, 4, 64, 32, 3, 1, 1, "random", 0, 0, True, False),
    (4, 2, 64, 64, 1, 31, 33, "random", 0, 0, False, True),
    (6, 2, 128, 32, 3, 777, 37, "random", 0, 0, True, True),
    (8, 2, 64, 256, 2, 1000, 256, "deep", 0, 0, True, True),
    (2, 2, 128, 32, 1, 65, 256, "chain", 0, 0, False, False),
    (3, 1, 64, 32, 2, 95, 64, "star", 0, 0, True, False),
    (100, 1, 128, 32, 2, 130, 9, "random", 0, 0, False, True),
    (32, 4, 128, 64, 2, 500, 63, "random", 0, 0, False, False),
    (6, 2, 128, 32, 2, 400, 40, "deep", 1, 0, False, False),
    (6, 2, 128, 32, 3, 400, 40, "chain", 7, 3, True, True),
    (8, 8, 64, 32, 3, 20, 64, "deep", 5, 28, True, False),
    (24, 8, 128, 64, 2, 2000, 32, "random", 333, 4, True, True),
    (6, 2, 64, 32, 2, 700, 21, "random", 64, 100, False, False),
    (6, 2, 64, 32, 2, 100, 21, "random", 5000, 500, True, False),
    (2, 1, 128, 64, 1, 9000, 70, "random", 0, 0, False, False),
    (6, 2, 128, 32, 2, 0, 30, "deep", 3, 2, False, True),
    (12, 2, 64, 32, 3, 2, 150, "deep", 4, 9, True, True),
    (24, 8, 64, 32, 20, 300, 33, "random", 0, 0, True, True),
    (24, 8, 128, 32, 20, 400, 43, "random", 100, 33, True, True),
    (128, 1, 64, 32, 2, 2500, 40, "random", 2200, 31, True, False),
    (32, 4, 128, 256, 1, 4100, 16, "chain", 0, 0, False, False),
]


@pytest.mark.parametrize("dtype", ALL_STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,nodes,kind,window,sinks,ragged,counts", TREES)
def test_tree(dtype, Hq, Hkv, D, Z, B, t, nodes, kind, window, sinks, ragged, counts):
    rng = np.random.default_rng(t * 1000 + nodes + window)
    steps = pick_steps(rng, t, B, ragged)
    n = np.resize([nodes, 0, max(1, nodes // 2)], B) if counts else np.full(B, nodes)
    parents = np.stack([tree_of(kind, nodes, rng) for _ in range(B)])
    q, K, V = normal(31, 1, (B, nodes, Hq, D), dtype), normal(31, 2, (B, t + nodes, Hkv, D), dtype), normal(31, 3, (B, t + nodes, Hkv, D), dtype)
    st = make_store(31, dtype, B, Hq, Hkv, D, Z, t + nodes - 1)
    write_lengths(st, K, V, steps + n)
    out = rows_of(dtype, np.full((B, nodes, Hq, D), UNTOUCHED))
    st.attend_tree(rows_of(dtype, q), out, ints(parents), t, ints(n) if counts else None, window, sinks, ints(steps) if ragged else None)
    got = np64(out)
    for b in range(B):
        assert (got[b, n[b]:] == UNTOUCHED).all()
        if n[b]:
            end = steps[b] + n[b]
            seen = sees_tree(steps[b], parents[b, :n[b]], window, sinks)
            near(dtype, got[b, :n[b]], q[b, :n[b]], K[b, :end], V[b, :end], seen)


@pytest.mark.parametrize("dtype", STORES)
def test_tree_with_parents_that_are_no_rows_before(dtype):
    """Anything but 0 .. i-1 is no parent: the node follows the last cached step."""
    B, Hq, Hkv, D, Z, t, nodes = 1, 4, 2, 64, 32, 50, 12
    parents = np.array([[5, 0, 2, -7, 3, 2 ** 31 - 1, 5, -2 ** 31, 8, 4, 11, 10]])
    q, K, V = normal(32, 1, (B, nodes, Hq, D)), normal(32, 2, (B, t + nodes, Hkv, D)), normal(32, 3, (B, t + nodes, Hkv, D))
    st = make_store(32, dtype, B, Hq, Hkv, D, Z, t + nodes - 1)
    write_lengths(st, K, V, [t + nodes])
    out = bf16(np.zeros((B, nodes, Hq, D)))
    st.attend_tree(bf16(q), out, ints(parents), t)
    within(np64(out)[0], *attention(q[0], kept(dtype, K[0]), kept(dtype, V[0]), sees_tree(t, parents[0], 0, 0)))
    clean = [p if 0 <= p < i else -1 for i, p in enumerate(parents[0])]
    positions = st.tree_positions(ints(parents), t).cpu().numpy()[0]
    np.testing.assert_array_equal(positions, t + depths(clean))


def test_a_chain_is_a_block_of_steps():
    B, Hq, Hkv, D, Z, t, nodes = 2, 6, 2, 128, 64, 333, 20
    q, K, V = normal(33, 1, (B, nodes, Hq, D)), normal(33, 2, (B, t + nodes, Hkv, D)), normal(33, 3, (B, t + nodes, Hkv, D))
    st = make_store(33, T.TEMPO_BF16, B, Hq, Hkv, D, Z, t + nodes - 1)
    write_lengths(st, K, V, [t + nodes] * B)
    tree, block = bf16(np.zeros(q.shape)), bf16(np.zeros(q.shape))
    st.attend_tree(bf16(q), tree, ints(np.tile(np.arange(nodes) - 1, (B, 1))), t)
    st.attend_block(bf16(q), block, t, nodes)
    for got in (tree, block):
        for b in range(B):
            within(np64(got)[b], *attention(q[b], K[b], V[b], sees_chain(t, nodes, 0, 0)))


@pytest.mark.parametrize("nodes,B,t,ragged", [(1, 1, 0, False), (17, 3, 100, True), (256, 2, 5, False), (255, 65, 2 ** 31 - 300, True)])
def test_positions_of_a_tree(nodes, B, t, ragged):
    rng = np.random.default_rng(nodes)
    parents = np.stack([tree_of(["random", "chain", "star", "deep"][b % 4], nodes, rng) for b in range(B)])
    steps = pick_steps(rng, t, B, ragged)
    steps[0] = t
    given = steps.copy()
    if ragged:
        given[0] = min(2 ** 31 - 1, t + 9)                     # t bounds the steps
        steps[-1], given[-1] = 0, -4
    positions = torch.empty((B, nodes), dtype=torch.int32, device=DEV)
    T.tempo_tree_positions(ints(parents), positions, B, nodes, t, ints(given) if ragged else None)
    np.testing.assert_array_equal(positions.cpu().numpy(), np.stack([steps[b] + depths(parents[b]) for b in range(B)]))


SINKS = [  # Hq, Hkv, D, Z, B, t, queries, window, sinks, ragged
    (24, 8, 128, 64, 2, 500, 1, 100, 4, False),
    (6, 2, 128, 32, 3, 0, 1, 1, 0, False),
    (6, 2, 128, 32, 3, 40, 1, 1, 5, True),
    (4, 4, 64, 32, 3, 700, 5, 33, 1, True),
    (8, 2, 64, 64, 2, 1000, 1, 64, 40, True),
    (8, 2, 64, 64, 2, 1000, 7, 64, 1000, True),
    (6, 2, 128, 32, 2, 300, 3, 290, 64, False),
    (6, 2, 128, 32, 2, 300, 3, 1000, 64, True),
    (100, 1, 128, 32, 2, 600, 2, 200, 33, False),
    (12, 4, 128, 256, 1, 5000, 40, 2500, 7, False),
    (2, 1, 64, 32, 1, 40000, 1, 20000, 70, False),
    (6, 2, 64, 32, 2, 95, 33, 32, 32, True),
    (8, 8, 128, 32, 40, 200, 1, 70, 3, True),
    (6, 2, 128, 32, 2, 150, 300, 90, 35, True),
    (8, 1, 64, 64, 3, 3000, 100, 600, 65, True),
    (4, 2, 128, 32, 2, 4500, 60, 4000, 2200, False),
]


@pytest.mark.parametrize("dtype", ALL_STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,queries,window,sinks,ragged", SINKS)
def test_steps_with_sinks(dtype, Hq, Hkv, D, Z, B, t, queries, window, sinks, ragged):
    rng = np.random.default_rng(t + queries)
    steps = pick_steps(rng, t, B, ragged)
    q, K, V = normal(41, 1, (B, queries, Hq, D), dtype), normal(41, 2, (B, t + queries, Hkv, D), dtype), normal(41, 3, (B, t + queries, Hkv, D), dtype)
    st = make_store(41, dtype, B, Hq, Hkv, D, Z, t + queries - 1)
    write_lengths(st, K, V, steps + queries)
    # keys that no step of the call sees may hold anything
    for b in range(B):
        dead = np.arange(steps[b] + queries)
        dead = dead[(dead >= sinks) & (dead <= steps[b] - window)]
        if dead.size and dead.size < 300:
            kv = T.make_kv(st.k_pool, st.v_pool, st.block_table[b:b + 1].contiguous(), st.num_blocks, st.max_blocks_per_seq, Z, Hkv, D, dtype)
            row = st.block_table[b:b + 1].contiguous()
            kv.block_table = row.data_ptr()
            nan = rows_of(dtype, np.full((1, dead.size, Hkv, D), np.nan))
            T.tempo_kv_append_block(kv, nan, nan, 1, int(dead[0]), None, int(dead.size))
            torch.cuda.synchronize()
    out = rows_of(dtype, np.zeros(q.shape))
    st.attend_sinks(rows_of(dtype, q), out, t, queries, window, sinks, ints(steps) if ragged else None)
    got = np64(out)
    for b in range(B):
        end = steps[b] + queries
        near(dtype, got[b], q[b], K[b, :end], V[b, :end], sees_chain(steps[b], queries, window, sinks))


@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,rows,window,sinks", [(6, 2, 128, 4, 2, 91, 7, 0, 0), (8, 2, 64, 8, 3, 700, 40, 33, 5), (3, 1, 128, 16, 1, 333, 1, 50, 30),
                                                              (4, 2, 64, 4, 2, 0, 3, 2, 1)])
def test_fp32_blocks_shorter_than_a_group(Hq, Hkv, D, Z, B, t, rows, window, sinks):
    dtype, rng = T.TEMPO_F32, np.random.default_rng(t)
    parents = np.stack([tree_of("random", rows, rng) for _ in range(B)])
    q, K, V = normal(43, 1, (B, rows, Hq, D), dtype), normal(43, 2, (B, t + rows, Hkv, D), dtype), normal(43, 3, (B, t + rows, Hkv, D), dtype)
    st = make_store(43, dtype, B, Hq, Hkv, D, Z, t + rows - 1)
    write_lengths(st, K, V, [t + rows] * B)
    tree, chain = rows_of(dtype, np.zeros(q.shape)), rows_of(dtype, np.zeros(q.shape))
    st.attend_tree(rows_of(dtype, q), tree, ints(parents), t, window=window, sinks=sinks)
    if window:
        st.attend_sinks(rows_of(dtype, q), chain, t, rows, window, sinks)
    for b in range(B):
        near(dtype, np64(tree)[b], q[b], K[b], V[b], sees_tree(t, parents[b], window, sinks))
        if window:
            near(dtype, np64(chain)[b], q[b], K[b], V[b], sees_chain(t, rows, window, sinks))


def angles(positions, D):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(D // 2) * 2 / D)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def to_bf16(x):
    return np64(bf16(x))


def to_rows(dtype, x):
    return np64(rows_of(dtype, x))


@pytest.mark.parametrize("dtype", ALL_STORES)
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,window,sinks,ragged", [(6, 2, 128, 32, 2, 50, 5, False), (4, 4, 64, 64, 3, 40, 33, True), (40, 2, 128, 32, 1, 9, 1, False)])
def test_an_endless_conversation_in_few_blocks(dtype, rope, Hq, Hkv, D, Z, B, window, sinks, ragged):
    """Steps one by one, each written by its own call, on a table that names the window's blocks in turn."""
    steps, lag = 260, np.array([0, 7, 70])[:B] if ragged else np.zeros(B, dtype=int)
    table, blocks = BlockStore.sinks_table(B, steps, Z, window, sinks)
    first, turn = T.tempo_sink_blocks(window, sinks, Z)
    assert blocks == B * (first + turn) and table.shape[1] > first + turn
    st = BlockStore(B, Hq, Hkv, D, Z, steps, dtype, device=DEV, num_blocks=blocks, block_table=table, fill="nan")
    q, K, V = normal(42, 1, (B, steps, Hq, D), dtype), normal(42, 2, (B, steps, Hkv, D), dtype), normal(42, 3, (B, steps, Hkv, D), dtype)
    c, s = angles(steps, D)
    st.set_rope(torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV))
    c, s = c.astype(np.float64), s.astype(np.float64)
    # (the store's keys are read back after their write, so that only the attention is compared with 64 bits)
    rows = np.zeros((B, steps, Hkv, D))
    out = rows_of(dtype, np.zeros((B, Hq, D)))
    for i in range(steps):
        at = i - lag
        live = np.maximum(at, 0)
        pick = np.arange(B), live
        st.step_sinks(rows_of(dtype, q[pick]), rows_of(dtype, K[pick]), rows_of(dtype, V[pick]), out, i, window, sinks, ints(live) if ragged else None, rope=rope)
        if rope:
            flat = to_rows(dtype, turned(K[pick], c[live][:, None], s[live][:, None]))
            if not ragged:
                k_back = np64(st.gather(i, 1)[0])[:, 0]
                assert np.abs(k_back - kept(dtype, flat)).max() <= (2.0 ** -3 if dtype == T.TEMPO_E4M3 else 2.0 ** -21 if dtype == T.TEMPO_F32 else 2.0 ** -7) * np.abs(flat).max()
                rows[:, i] = k_back
            else:
                rows[pick] = kept(dtype, flat)
        else:
            rows[pick] = kept(dtype, K[pick])
        if i in (0, 1, 8, 31, 32, 63, 64, 65, 100, 127, 128, 200, 255, 259):
            got = np64(out)
            for b in range(B):
                p = live[b]
                qb = to_rows(dtype, turned(q[b, p], c[p], s[p])) if rope else q[b, p]
                o, size = attention(qb[None], rows[b, :p + 1], kept(dtype, V[b, :p + 1]), sees_chain(p, 1, window, sinks))
                if dtype == T.TEMPO_F32:
                    within_fp32(got[b][None], o, size, qb[None], rows[b, :p + 1], turns=2 * rope)
                elif not rope:
                    within(got[b][None], o, size)
                else:  # a rounding of q or k that goes the other way: a step of it in one of D products each
                    assert np.abs(got[b][None] - o).max() <= 0.05 * np.abs(size).max()


PROMPTS = [  # Hq, Hkv, D, Z, B, t, count, window, sinks, counts
    (6, 2, 128, 32, 2, 0, 1, 10, 2, False),
    (6, 2, 128, 64, 2, 0, 200, 50, 4, False),
    (24, 8, 128, 64, 3, 0, 333, 100, 40, True),
    (4, 4, 64, 32, 2, 17, 150, 32, 1, True),
    (8, 2, 64, 256, 1, 1000, 90, 700, 33, False),
    (32, 4, 128, 32, 1, 100, 130, 1, 1, False),
    (3, 1, 128, 32, 2, 45, 300, 5000, 4, True),
    (100, 1, 64, 32, 1, 0, 40, 16, 8, False),
    (8, 2, 128, 64, 1, 0, 1100, 256, 0, False),
]


@pytest.mark.parametrize("dtype", ALL_STORES)
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,count,window,sinks,counts", PROMPTS)
def test_prompts_with_sinks(dtype, Hq, Hkv, D, Z, B, t, count, window, sinks, counts):
    n = np.array([count, 0, count // 3])[:B] if counts else np.full(B, count)
    q, K, V = normal(51, 1, (B, count, Hq, D), dtype), normal(51, 2, (B, t + count, Hkv, D), dtype), normal(51, 3, (B, t + count, Hkv, D), dtype)
    st = make_store(51, dtype, B, Hq, Hkv, D, Z, t + count - 1)
    write_lengths(st, K, V, [t] * B)
    before = st.k_pool.clone(), st.v_pool.clone()
    out = rows_of(dtype, np.full(q.shape, UNTOUCHED))
    st.prefill_sinks(rows_of(dtype, q), rows_of(dtype, K[:, t:]), rows_of(dtype, V[:, t:]), out, t, count, window, sinks, ints(n) if counts else None)
    got = np64(out)
    for b in range(B):
        assert (got[b, n[b]:] == UNTOUCHED).all()
        if n[b]:
            end = t + n[b]
            near(dtype, got[b, :n[b]], q[b, :n[b]], K[b, :end], V[b, :end], sees_chain(t, n[b], window, sinks))
    # the store holds the rows, and nothing else changed
    k_back, v_back = (np64(x) for x in st.gather(0, t + count))
    for b in range(B):
        np.testing.assert_array_equal(k_back[b, :t + n[b]], kept(dtype, K[b, :t + n[b]]))
        np.testing.assert_array_equal(v_back[b, :t + n[b]], kept(dtype, V[b, :t + n[b]]))
    if counts and B > 1:
        mine = st.block_table[1].long()
        if dtype != T.TEMPO_E4M3:
            for old, new in zip(before, (st.k_pool, st.v_pool)):
                assert torch.equal(old[mine].view(torch.uint8), new[mine].view(torch.uint8))


@pytest.mark.parametrize("dtype", STORES)
def test_a_rotated_prompt_is_the_rotated_rows_prompt(dtype):
    Hq, Hkv, D, Z, B, t, count, window, sinks = 6, 2, 128, 32, 2, 21, 100, 40, 5
    q, K, V = normal(52, 1, (B, count, Hq, D)), normal(52, 2, (B, count, Hkv, D)), normal(52, 3, (B, count, Hkv, D))
    c, s = (torch.from_numpy(x).to(DEV) for x in angles(t + count, D))
    got = []
    for fused in (True, False):
        st = make_store(52, dtype, B, Hq, Hkv, D, Z, t + count - 1)
        st.k_pool.zero_(), st.v_pool.zero_()
        st.set_rope(c, s)
        out = bf16(np.zeros(q.shape))
        if fused:
            st.prefill_sinks(bf16(q), bf16(K), bf16(V), out, t, count, window, sinks, rope=True)
        else:
            qr = bf16(q)
            st.rope_append_block(bf16(K), bf16(V), t, count)
            positions = ints(np.tile(t + np.arange(count), (B, 1)))
            T.tempo_rope_rotate_at(st.rope, None, positions, qr, qr, T.TEMPO_BF16, B, count, Hq)
            st.attend_sinks(qr, out, t, count, window, sinks)
        got.append((np64(out), [x.view(torch.uint8).clone() for x in (st.k_pool, st.v_pool)]))
    for a, b in zip(got[0][1], got[1][1]):
        assert torch.equal(a, b)
    np.testing.assert_array_equal(got[0][0], got[1][0])


@pytest.mark.parametrize("dtype", ALL_STORES)
def test_a_drafting_decoder(dtype):
    """Three layers, four steps of drafting: rows placed at their positions, answered, the accepted path kept.  The store then holds, and
    the next steps answer from, what a decoder without drafts would have."""
    half_step = 2.0 ** -8 if dtype != T.TEMPO_F32 else 2.0 ** -21  # of a turned element, against the largest (fp32: 2 roundings of a pair)
    layers, B, Hq, Hkv, D, Z, t0, nodes = 3, 2, 6, 2, 128, 32, 45, 14
    rng = np.random.default_rng(6)
    room = t0 + 200
    c, s = angles(room, D)
    tables = torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV)
    c, s = c.astype(np.float64), s.astype(np.float64)
    stores = [make_store(60, dtype, B, Hq, Hkv, D, Z, room - 1) for _ in range(layers)]
    for st in stores:
        st.block_table = stores[0].block_table
        st.kv.block_table = stores[0].block_table.data_ptr()
        st.set_rope(*tables)
    K = [normal(61 + i, 2, (B, t0, Hkv, D), dtype) for i in range(layers)]
    V = [normal(61 + i, 3, (B, t0, Hkv, D), dtype) for i in range(layers)]
    for i, st in enumerate(stores):
        st.rope_append_at(ints(np.tile(np.arange(t0)[:, None], (B, 1, 1))), rows_of(dtype, K[i]), rows_of(dtype, V[i]), 0)
    rows = [[np64(x) for x in st.gather(0, t0)] for st in stores]   # what the layers' sequences hold
    rows = [[[k[b] for b in range(B)], [v[b] for b in range(B)]] for k, v in rows]
    steps = np.full(B, t0)
    for turn in range(4):
        parents = np.stack([tree_of("random", nodes, rng) for _ in range(B)])
        top = int(steps.max())
        positions = stores[0].tree_positions(ints(parents), top, ints(steps))
        np.testing.assert_array_equal(positions.cpu().numpy(), np.stack([steps[b] + depths(parents[b]) for b in range(B)]))
        paths = [ancestors(parents[b], int(rng.integers(0, nodes)))[::-1] for b in range(B)]
        for i, st in enumerate(stores):
            q, k, v = (normal(70 + 10 * turn + i, w, (B, nodes, h, D), dtype) for w, h in ((1, Hq), (2, Hkv), (3, Hkv)))
            turned_q, out = rows_of(dtype, q), rows_of(dtype, np.zeros(q.shape))
            st.rope_append_at(positions[..., None].contiguous(), rows_of(dtype, k), rows_of(dtype, v), top, turned_q, turned_q, ints(steps))
            st.attend_tree(turned_q, out, ints(parents), top, t_per_seq=ints(steps))
            got = np64(out)
            for b in range(B):
                p = steps[b] + depths(parents[b])
                k_now = kept(dtype, to_rows(dtype, turned(k[b], c[p][:, None], s[p][:, None])))
                q_now = np64(turned_q)[b]
                assert np.abs(q_now - turned(q[b], c[p][:, None], s[p][:, None])).max() <= half_step * 1.01 * np.abs(q_now).max()
                keys, values = np.concatenate([rows[i][0][b], k_now]), np.concatenate([rows[i][1][b], kept(dtype, v[b])])
                o, size = attention(q_now, keys, values, sees_tree(int(steps[b]), parents[b], 0, 0))
                if dtype == T.TEMPO_F32:
                    within_fp32(got[b], o, size, q_now, keys, turns=1)
                else:
                    assert np.abs(got[b] - o).max() <= 0.05 * size.max()  # (a key's rounding that goes the other way)
                for which, new in ((0, k_now), (1, kept(dtype, v[b]))):
                    rows[i][which][b] = np.concatenate([rows[i][which][b], new[paths[b]]])
        longest = max(len(x) for x in paths)
        path = np.array([x + [-1] * (longest - len(x)) for x in paths])
        stores[0].keep(ints(path), top, nodes, ints(steps), layers=stores)
        steps = steps + np.array([len(x) for x in paths])
        for i, st in enumerate(stores):
            k_back, v_back = (np64(x) for x in st.gather(0, int(steps.max())))
            for b in range(B):
                np.testing.assert_array_equal(v_back[b, :steps[b]], rows[i][1][b])
                assert np.abs(k_back[b, :steps[b]] - rows[i][0][b]).max() <= (0.13 if dtype == T.TEMPO_E4M3 else 2 * half_step) * np.abs(rows[i][0][b]).max()
                rows[i][0][b] = k_back[b, :steps[b]].copy()


@pytest.mark.parametrize("dtype", ALL_STORES)
def test_on_another_stream_and_captured(dtype):
    """A tree and a step with sinks in one graph, replayed with other inputs, steps and trees; eager work between the replays."""
    B, Hq, Hkv, D, Z, t, nodes, window, sinks = 2, 6, 2, 128, 32, 900, 24, 300, 4
    K, V = normal(81, 2, (B, t + nodes, Hkv, D), dtype), normal(81, 3, (B, t + nodes, Hkv, D), dtype)
    st = make_store(81, dtype, B, Hq, Hkv, D, Z, t + nodes - 1)
    st.append_block(rows_of(dtype, K), rows_of(dtype, V), 0, t + nodes)
    rng = np.random.default_rng(8)
    q = torch.zeros((B, nodes, Hq, D), dtype=rows_of(dtype, 0.0).dtype, device=DEV)
    parents, steps = ints(np.full((B, nodes), -1)), ints(np.full(B, t))
    q1 = torch.zeros((B, Hq, D), dtype=rows_of(dtype, 0.0).dtype, device=DEV)
    out, out1 = torch.zeros_like(q), torch.zeros_like(q1)

    def both(a, b):
        st.attend_tree(q, a, parents, t, t_per_seq=steps)
        st.attend_sinks(q1, b, t, 1, window, sinks, steps)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(out, out1)
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out, out1)
    for turn in range(4):
        q.copy_(rows_of(dtype, normal(82 + turn, 1, q.shape, dtype)))
        q1.copy_(rows_of(dtype, normal(82 + turn, 4, q1.shape, dtype)))
        parents.copy_(ints(np.stack([tree_of("random", nodes, rng) for _ in range(B)])))
        steps.copy_(ints(np.array([t, 40 + 200 * turn])))
        graph.replay()
        torch.cuda.synchronize()
        eager, eager1 = torch.zeros_like(out), torch.zeros_like(out1)
        both(eager, eager1)
        assert torch.equal(out, eager) and torch.equal(out1, eager1)
        P = parents.cpu().numpy()
        for b, at in enumerate(steps.cpu().numpy()):
            end = at + nodes
            near(dtype, np64(out)[b], np64(q)[b], K[b, :end], V[b, :end], sees_tree(int(at), P[b], 0, 0))
            near(dtype, np64(out1)[b][None], np64(q1)[b][None], K[b, :at + 1], V[b, :at + 1], sees_chain(int(at), 1, window, sinks))


def test_steps_beyond_their_bound_and_below_zero():
    """t_per_seq is cut to 0 .. t."""
    B, Hq, Hkv, D, Z, t, window, sinks = 3, 4, 2, 64, 32, 100, 30, 3
    q, K, V = normal(91, 1, (B, 1, Hq, D)), normal(91, 2, (B, t + 1, Hkv, D)), normal(91, 3, (B, t + 1, Hkv, D))
    st = make_store(91, T.TEMPO_BF16, B, Hq, Hkv, D, Z, t)
    write_lengths(st, K, V, [t + 1] * B)
    out = bf16(np.zeros(q.shape))
    st.attend_sinks(bf16(q), out, t, 1, window, sinks, ints([t + 50, -5, 2 ** 31 - 1]))
    for b, at in enumerate((t, 0, t)):
        within(np64(out)[b], *attention(q[b], K[b, :at + 1], V[b, :at + 1], sees_chain(at, 1, window, sinks)))


@pytest.mark.parametrize("dtype", STORES)
def test_values_that_nobody_sees_and_large_ones(dtype):
    """Infinities and NaN in slots that no row sees do not show; logits of any size do not overflow."""
    B, Hq, Hkv, D, Z, t, nodes = 1, 4, 1, 64, 32, 70, 6
    q, K, V = normal(95, 1, (B, nodes, Hq, D)) * 40, normal(95, 2, (B, t + nodes, Hkv, D)) * 100, normal(95, 3, (B, t + nodes, Hkv, D))
    q, K = to_bf16(q), to_bf16(K)
    st = make_store(95, dtype, B, Hq, Hkv, D, Z, t + nodes + 20)
    write_lengths(st, K, V, [t + nodes])
    bad = bf16(np.full((B, 10, Hkv, D), np.inf))
    st.append_block(bad, bad, t + nodes, 10)
    parents = np.array([[-1, 0, 0, 2, -1, 4]])
    out = bf16(np.zeros(q.shape))
    st.attend_tree(bf16(q), out, ints(parents), t)
    o, size = attention(q[0], kept(dtype, K[0]), kept(dtype, V[0]), sees_tree(t, parents[0], 0, 0))
    # logits of some ten thousand, in fp32: their rounding, 2^-24 of D products' sum each, moves a weight by that much
    top = np.abs(np.einsum("nhd,td->nht", np.abs(q[0]), np.abs(kept(dtype, K[0]))[:, 0])).max() / 8.0
    slack = 4 * D * 2.0 ** -24 * top
    assert np.abs(np64(out)[0] - o).max() <= (1.03 * 2.0 ** -8 * 3 + 2 * slack) * np.abs(V).max()


@pytest.mark.parametrize("dtype", ALL_STORES)
@pytest.mark.parametrize("seed", range(24))
def test_drawn_calls(dtype, seed):
    """Trees, steps and prompts of any shape."""
    rng = np.random.default_rng(1000 + seed)
    pick = lambda *x: x[int(rng.integers(0, len(x)))]  # noqa: E731
    Hkv, G, D, B = pick(1, 2, 3, 8), pick(1, 2, 3, 4, 5, 8, 16, 17, 33, 128), pick(64, 128), pick(1, 2, 3, 7)
    Z, t = pick(32, 64, 128), int(2 ** rng.uniform(0, 9.5)) - 1
    rows = min(int(2 ** rng.uniform(0, 8.1)), max(1, 1200 // (G * Hkv)))
    window, sinks = pick(1, 2, 33, int(2 ** rng.uniform(0, 10))), pick(0, 1, 4, int(2 ** rng.uniform(0, 8)))
    ragged, counts, Hq = rng.random() < 0.5, rng.random() < 0.5, G * Hkv
    n = rng.integers(0, rows + 1, B) if counts else np.full(B, rows)
    q, K, V = normal(seed, 1, (B, rows, Hq, D), dtype), normal(seed, 2, (B, t + rows, Hkv, D), dtype), normal(seed, 3, (B, t + rows, Hkv, D), dtype)

    def check(got, seen, steps, n):
        for b in range(B):
            assert (got[b, n[b]:] == UNTOUCHED).all()
            if n[b]:
                end = steps[b] + n[b]
                near(dtype, got[b, :n[b]], q[b, :n[b]], K[b, :end], V[b, :end], seen(b))

    st = make_store(seed, dtype, B, Hq, Hkv, D, Z, t + rows - 1)
    steps = pick_steps(rng, t, B, ragged)
    parents = np.stack([tree_of(pick("random", "chain", "star", "deep"), rows, rng) for _ in range(B)])
    write_lengths(st, K, V, steps + n)
    out = rows_of(dtype, np.full(q.shape, UNTOUCHED))
    for w, s in ((0, 0), (window, sinks)):
        out.fill_(UNTOUCHED)
        st.attend_tree(rows_of(dtype, q), out, ints(parents), t, ints(n) if counts else None, w, s, ints(steps) if ragged else None)
        check(np64(out), lambda b: sees_tree(steps[b], parents[b, :n[b]], w, s), steps, n)
    write_lengths(st, K, V, steps + rows)
    st.attend_sinks(rows_of(dtype, q), out, t, rows, window, sinks, ints(steps) if ragged else None)
    check(np64(out), lambda b: sees_chain(steps[b], rows, window, sinks), steps, np.full(B, rows))
    st = make_store(seed, dtype, B, Hq, Hkv, D, Z, t + rows - 1)
    write_lengths(st, K, V, np.full(B, t))
    out.fill_(UNTOUCHED)
    st.prefill_sinks(rows_of(dtype, q), rows_of(dtype, K[:, t:]), rows_of(dtype, V[:, t:]), out, t, rows, window, sinks, ints(n) if counts else None)
    check(np64(out), lambda b: sees_chain(t, n[b], window, sinks), np.full(B, t), n)


def framed(n, dtype):
    """A tensor of n elements between two frames of 4096, and a check that the frames are as they were."""
    whole = torch.full((n + 8192,), 119, dtype=torch.uint8, device=DEV) if dtype == torch.uint8 else torch.full((n + 8192,), -9.0, dtype=dtype, device=DEV)
    before = whole.clone()

    def intact():
        assert torch.equal(whole[:4096], before[:4096]) and torch.equal(whole[-4096:], before[-4096:])
    return whole[4096:4096 + n], intact


@pytest.mark.parametrize("dtype", ALL_STORES)
@pytest.mark.parametrize("Hq,Hkv,D,B,t,rows,window,sinks", [
    (24, 8, 128, 2, 700, 1, 300, 4), (24, 8, 128, 3, 333, 8, 100, 5), (32, 8, 64, 1, 2500, 13, 1000, 33), (32, 4, 128, 2, 900, 41, 500, 4),
    (32, 4, 64, 1, 3000, 23, 2000, 0), (16, 16, 64, 20, 90, 30, 60, 2), (6, 2, 128, 2, 40, 256, 77, 3), (128, 1, 64, 1, 1500, 3, 900, 31),
])
def test_nothing_is_written_beside_answers_workspace_and_rows(dtype, Hq, Hkv, D, B, t, rows, window, sinks):
    """Exact workspaces and answers between frames; blocks of no sequence and slots behind the rows stay."""
    rng = np.random.default_rng(t)
    st = make_store(97, dtype, B, Hq, Hkv, D, 64, t + rows - 1)
    K, V = normal(97, 2, (B, t, Hkv, D), dtype), normal(97, 3, (B, t, Hkv, D), dtype)
    write_lengths(st, K, V, [t] * B)
    q, k, v = (rows_of(dtype, normal(98, w, (B, rows, h, D), dtype)) for w, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    parents = ints(np.stack([tree_of("random", rows, rng) for _ in range(B)]))
    out, out_intact = framed(q.numel(), q.dtype)
    out = out.view(q.shape)
    pools = st.k_pool.clone(), st.v_pool.clone()
    n = T.tempo_prefill_sinks_workspace_bytes(st.kv, B, Hq, t + rows - 1)
    n = min(n, T.tempo_attn_sinks_workspace_bytes(st.kv, B, Hq, rows, t, window, sinks))  # (of the same steps: as much is needed)
    ws, ws_intact = framed(n, torch.uint8)
    assert ws.data_ptr() % 256 == 0
    T.tempo_prefill_sinks(st.kv, q, k, v, out, B, Hq, t, rows, None, window, sinks, st.scale, ws, n)
    out_intact(), ws_intact()
    first = out.clone()
    written = st.k_pool.clone(), st.v_pool.clone()
    T.tempo_attn_sinks(st.kv, q, out, B, Hq, rows, t, None, window, sinks, st.scale, ws, n)
    out_intact(), ws_intact()
    if rows > 1:  # (a single step's row is patched in as it is written, with the same bits)
        assert torch.equal(out, first)
    n = T.tempo_attn_tree_workspace_bytes(st.kv, B, Hq, rows, t, window, sinks)
    ws, ws_intact = framed(n, torch.uint8)
    T.tempo_attn_tree(st.kv, q, out, parents, None, B, Hq, rows, t, None, window, sinks, st.scale, ws, n)
    out_intact(), ws_intact()
    for now, then in zip((st.k_pool, st.v_pool), written):  # attention writes no row
        assert torch.equal(now.view(torch.uint8), then.view(torch.uint8))
    # blocks that no sequence has, and those that hold none of the rows
    changed = torch.ones(st.num_blocks, dtype=torch.bool, device=DEV)
    changed[st.block_table[:, t // 64:(t + rows - 1) // 64 + 1].flatten().long()] = False
    for now, then in zip((st.k_pool, st.v_pool), pools):
        codes = st.num_blocks * Hkv * 64 * D if dtype == T.TEMPO_E4M3 else now.numel()
        a, b = (x.flatten()[:codes].view(st.num_blocks, -1).view(torch.uint8) for x in (now, then))
        assert torch.equal(a[changed], b[changed])
        if dtype == T.TEMPO_E4M3:
            a, b = (x.flatten()[codes:].view(st.num_blocks, -1) for x in (now, then))
            assert torch.equal(a[changed], b[changed])


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,B,ragged", [(16, 8, 128, 200, False), (16, 8, 128, 230, True), (136, 8, 128, 180, False), (32, 8, 64, 330, False), (32, 8, 64, 260, True)])
def test_many_workgroups_of_few_groups(dtype, Hq, Hkv, D, B, ragged):
    """One or two wavefronts to a workgroup: steps that write their row, trees."""
    rng = np.random.default_rng(B)
    t, window, sinks, nodes = 130, 90, 3, 2
    steps = pick_steps(rng, t, B, ragged)
    st = make_store(99, dtype, B, Hq, Hkv, D, 32, t + nodes)
    K, V = normal(99, 2, (B, t + nodes, Hkv, D)), normal(99, 3, (B, t + nodes, Hkv, D))
    st.append_block(bf16(K), bf16(V), 0, t + nodes)
    # the step's row is written anew
    k, v, q = normal(100, 2, (B, Hkv, D)), normal(100, 3, (B, Hkv, D)), normal(100, 1, (B, Hq, D))
    out = bf16(np.zeros(q.shape))
    st.step_sinks(bf16(q), bf16(k), bf16(v), out, t, window, sinks, ints(steps) if ragged else None)
    got, some = np64(out), [0, 1, B - 1] + [int(b) for b in rng.integers(0, B, 7)]
    for b in some:
        K[b, steps[b]], V[b, steps[b]] = k[b], v[b]
        end = steps[b] + 1
        near(dtype, got[b][None], q[b][None], K[b, :end], V[b, :end], sees_chain(steps[b], 1, window, sinks))
    k_back, v_back = (np64(x) for x in st.gather(0, t + 1))
    for b in some:
        np.testing.assert_array_equal(k_back[b], kept(dtype, K[b, :t + 1]))
        np.testing.assert_array_equal(v_back[b], kept(dtype, V[b, :t + 1]))
    parents = np.tile([[-1, 0]], (B, 1))
    parents[::2, 1] = -1
    q = normal(101, 1, (B, nodes, Hq, D))
    out = bf16(np.zeros(q.shape))
    st.attend_tree(bf16(q), out, ints(parents), t, t_per_seq=ints(steps) if ragged else None)
    got = np64(out)
    for b in some:
        end = steps[b] + nodes
        near(dtype, got[b], q[b], K[b, :end], V[b, :end], sees_tree(steps[b], parents[b], 0, 0))


@pytest.mark.parametrize("dtype", STORES)
@pytest.mark.parametrize("Hq,Hkv,D,B,count,window", [(16, 8, 128, 6, 900, 40), (8, 8, 64, 8, 1300, 60), (40, 8, 128, 3, 500, 20), (32, 8, 64, 2, 2500, 30)])
def test_long_prompts_of_short_windows(dtype, Hq, Hkv, D, B, count, window):
    st = make_store(103, dtype, B, Hq, Hkv, D, 64, count - 1)
    q, K, V = normal(103, 1, (B, count, Hq, D)), normal(103, 2, (B, count, Hkv, D)), normal(103, 3, (B, count, Hkv, D))
    out = bf16(np.full(q.shape, UNTOUCHED))
    n = np.full(B, count)
    n[1] = count // 2 + 1
    st.prefill_sinks(bf16(q), bf16(K), bf16(V), out, 0, count, window, 4, ints(n))
    got = np64(out)
    for b in (0, 1, B - 1):
        assert (got[b, n[b]:] == UNTOUCHED).all()
        for first in (0, n[b] // 2, n[b] - 150):  # (rows 150 at a time: what they see lies among the sinks and the keys near them)
            rows = np.arange(first, min(first + 150, n[b]))
            seen = sees_chain(0, int(rows[-1]) + 1, window, 4)[rows]
            near(dtype, got[b, rows], q[b, rows], K[b, :rows[-1] + 1], V[b, :rows[-1] + 1], seen)


@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,rows,window,sinks,ragged", [
    (6, 2, 128, 32, 2, 50, 12, 0, 0, False), (4, 4, 64, 4, 3, 333, 40, 20, 5, True), (24, 8, 128, 64, 2, 3000, 8, 600, 70, True),
    (16, 1, 64, 32, 1, 0, 60, 7, 0, False), (1, 1, 128, 8, 1, 100, 33, 3, 110, False)])
def test_fp32_values_that_are_not_finite_show_only_where_they_are_seen(Hq, Hkv, D, Z, B, t, rows, window, sinks, ragged):
    """NaN and infinities among the values that some rows of a tree, a block or a prompt see: the other rows keep their bits, and so do the
    dims of those rows that hold none."""
    dtype, rng = T.TEMPO_F32, np.random.default_rng(t + rows)
    end, steps = t + rows, pick_steps(rng, t, B, ragged)
    parents = np.stack([tree_of("random", rows, rng) for _ in range(B)])
    q, K, V = normal(44, 1, (B, rows, Hq, D), dtype), normal(44, 2, (B, end, Hkv, D), dtype), normal(44, 3, (B, end, Hkv, D), dtype)
    worse = V.copy()
    for b in range(B):
        last = steps[b] + rows
        for j in {int(steps[b]), int(steps[b]) + rows // 2, last - 1, max(0, int(steps[b]) - max(1, window - rows // 3)), int(rng.integers(0, last))}:
            worse[b, j, rng.integers(0, Hkv), rng.integers(0, D, 3)] = np.array([np.nan, np.inf, -np.inf])[rng.permutation(3)]
    answers = []
    for values in (V, worse):
        st = make_store(44, dtype, B, Hq, Hkv, D, Z, end - 1)
        write_lengths(st, K, values, steps + rows)
        tree, block = rows_of(dtype, np.zeros(q.shape)), rows_of(dtype, np.zeros(q.shape))
        st.attend_tree(rows_of(dtype, q), tree, ints(parents), t, None, window, sinks, ints(steps) if ragged else None)
        answers.append([np64(tree)])
        if window:
            st.attend_sinks(rows_of(dtype, q), block, t, rows, window, sinks, ints(steps) if ragged else None)
            answers[-1].append(np64(block))
        if window and not ragged:
            st.prefill_sinks(rows_of(dtype, q), rows_of(dtype, K[:, t:]), rows_of(dtype, values[:, t:]), block, t, rows, window, sinks)
            answers[-1].append(np64(block))
    for which, (clean, got) in enumerate(zip(*answers)):
        for b in range(B):
            last = steps[b] + rows
            seen = sees_tree(int(steps[b]), parents[b], window, sinks) if which == 0 else sees_chain(int(steps[b]), rows, window, sinks)
            hit = seen.astype(float) @ (~np.isfinite(worse[b, :last])).reshape(last, -1) > 0     # [rows][Hkv * D]
            hit = hit.reshape(rows, Hkv, 1, D).repeat(Hq // Hkv, 2).reshape(rows, Hq, D)
            assert hit.any() and not hit.all() and not np.isfinite(got[b][hit]).any()
            np.testing.assert_array_equal(got[b][~hit], clean[b][~hit])
