"""The 8-bit block store on the GPU: what is written and read back, exactly; attention over it against the
fp64 oracle on the values that the codes stand for.

Tolerance of an answer o = sum p_j v_j / sum p_j: the kernel rounds each weight p_j to bf16, at most 2^-8 of it, and
divides by the sum of the rounded ones, so o moves by at most 2^-8 (A + |o|), A = sum p_j |v_j| / sum p_j, and the
result is rounded to bf16, 2^-8 |o|.  What fp32 adds: a logit x is off by at most (D + 4) 2^-24 sum |q_d k_d| scale
(D products, the scale, log2 e), below 1e-4 for the N(0, 1) inputs here (sum |q k| scale below 12), which is a
relative error of a weight below 1e-4; sums of n weights add n 2^-24 at the most.  Together 2^-8 (A + 2 |o|) and
3% of it for the fp32 part (1e-4 / 2^-8)."""
import numpy as np
import pytest
import torch

from e4m3_reference import CODES, held, scale_exponents
from oracle import tempo_oracle as oracle
from paper_2501_05408_amd import synth
from paper_2501_05408_amd import tempo as T
from paper_2501_05408_amd.store import BlockStore

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E4M3 = T.TEMPO_E4M3


def np64(x):
    return x.detach().float().cpu().numpy().astype(np.float64)


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).to(DEV)


def ints(x):
    return torch.from_numpy(np.asarray(x).astype(np.int32)).to(DEV)


def normal(seed, which, shape):
    return synth.normal_as(seed, which, shape, "bf16").astype(np.float64)


def make_store(seed, B, Hq, Hkv, D, Z, max_t, ring=0):
    """A poisoned store with a random block table and a few blocks that belong to nobody."""
    columns = ring if ring else max_t // Z + 1
    n = B * columns + 3
    table = torch.from_numpy(synth.permutation(seed, 77, n)[:B * columns].reshape(B, columns).copy())
    return BlockStore(B, Hq, Hkv, D, Z, max_t, E4M3, device=DEV, num_blocks=n, block_table=table, fill="nan", ring_blocks=ring)


def assert_attention(got, q, K, V, t, window, scale, what):
    """got [B][Hq][D] against the oracle over K, V [B][T][Hkv][D] (what the store holds)."""
    ref = oracle.attend(q, K, V, t, window, scale)
    size = oracle.attend(q, K, np.abs(V), t, window, scale)
    err = np.abs(np64(got) - ref)
    tol = 1.03 * 2.0 ** -8 * (size + 2 * np.abs(ref))
    assert np.isfinite(err).all() and (err <= tol).all(), f"{what}: {np.nanmax(err / tol):.3f} of the tolerance"


# ---- the rows ---------------------------------------------------------------------------------------

def rows_of_every_value(D):
    """All bf16 values: in rows of neighbours (one exponent a row), and mixed with others of up to 2^30 times the size."""
    bits = np.arange(65536, dtype=np.uint16)
    mixed = synth.permutation(3, 1, 65536).astype(np.uint16)
    near = np.where((mixed & 0x7F80) > 0x7000, mixed, (mixed & 0x87FF) | 0x3800).astype(np.uint16)  # exponents of a middle range
    x = torch.from_numpy(np.concatenate([bits, mixed, near]).view(np.int16)).view(torch.bfloat16)
    return x.double().numpy().reshape(-1, D)


@pytest.mark.parametrize("D", [64, 128])
def test_every_bf16_value_is_quantised_as_defined(D):
    rows = rows_of_every_value(D)                                    # [n][D]
    Hkv, Z = 4, 64
    n = rows.shape[0] // Hkv
    K = rows.reshape(1, n, Hkv, D)
    V = K[:, ::-1].copy()
    st = make_store(1, 1, Hkv, Hkv, D, Z, n - 1)
    st.append_block(bf16(K), bf16(V), 0, n)
    k, v = st.gather(0, n)
    for got, x in ((k, K), (v, V)):
        np.testing.assert_array_equal(np64(got), held(x))
    # the codes and scale bytes themselves, where the header says they are
    kp, vp, table = st.k_pool.cpu().numpy(), st.v_pool.cpu().numpy(), st.block_table.cpu().numpy()
    rng = np.random.default_rng(5)
    for _ in range(300):
        j, h, d = int(rng.integers(n)), int(rng.integers(Hkv)), int(rng.integers(D))
        for which, pool, x in ((0, kp, K), (1, vp, V)):
            e = scale_exponents(x[0, j, h])
            at = T.tempo_kv_scale_offset(st.kv, which, int(table[0, j // Z]), h, j % Z)
            assert pool[at] == e + 127
            code = pool[T.tempo_kv_element_offset(st.kv, which, int(table[0, j // Z]), h, j % Z, d)]
            np.testing.assert_array_equal(CODES[code], held(x[0, j, h])[d] / 2.0 ** float(e))


@pytest.mark.parametrize("by_rows", [False, True])
@pytest.mark.parametrize("E", [16, 17, 60, 126, 127, 128, 200, 246, 247])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_every_size_beside_a_rows_largest(D, E, by_rows):
    """Rows without NaN: every mantissa and sign from the largest exponent of a scale down to what rounds to 0, each row with
    one element that fixes its scale."""
    top = E + 8 if E < 247 else 254                   # largest exponent field of a row with this scale byte
    bits = np.array([(s << 15) | (x << 7) | m for s in (0, 1) for x in range(max(0, top - 21), top + 1) for m in range(128)
                     if x < top or m <= (0x60 if E < 247 else 0x7F)], dtype=np.uint16)
    bits = bits[synth.permutation(9, 1, len(bits))]
    bits = np.concatenate([bits, bits[:-len(bits) % (D - 1)]]).reshape(-1, D - 1)
    most = np.full((len(bits), 1), (top << 7) | (0x60 if E < 247 else 0x7F), dtype=np.uint16)
    rows = np.concatenate([bits[:, :D // 3], most, bits[:, D // 3:]], axis=1)
    x = torch.from_numpy(rows.view(np.int16)).view(torch.bfloat16).double().numpy()
    assert (scale_exponents(x) == E - 127).all()
    K = x.reshape(1, -1, 1, D)
    V = K[:, ::-1].copy()
    n = K.shape[1]
    st = make_store(2, 1, 1, 1, D, 32, n - 1)
    if by_rows:                                       # (a call with steps of its own for each sequence writes row by row)
        T.tempo_kv_append_block(st.kv, bf16(K), bf16(V), 1, 0, torch.zeros(1, dtype=torch.int32, device=DEV), n)
    else:
        st.append_block(bf16(K), bf16(V), 0, n)
    k, v = st.gather(0, n)
    np.testing.assert_array_equal(np64(k), held(K))
    np.testing.assert_array_equal(np64(v), held(V))


@pytest.mark.parametrize("D", [64, 128])
def test_every_code_and_scale_is_read_back(D):
    """The 256 codes under every scale a row can have, put into the pools by hand."""
    Z, scales = 32, np.arange(16, 248)
    st = BlockStore(1, 1, 1, D, Z, len(scales) * 256 // D - 1, E4M3, device=DEV)
    rows = len(scales) * 256 // D
    values = (CODES[None, :] * 2.0 ** (scales[:, None] - 127.0)).reshape(rows, D)
    values = np.where(np.abs(values) >= 2.0 ** 128, np.copysign(np.inf, values), values)  # (no row is written so)
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8), (len(scales), 256)).reshape(rows, D)
    for which, pool in ((0, st.k_pool), (1, st.v_pool)):
        raw = np.zeros(pool.numel(), dtype=np.uint8)
        for j in range(rows):
            raw[T.tempo_kv_scale_offset(st.kv, which, j // Z, 0, j % Z)] = scales[j * D // 256]
            for d in range(D):
                raw[T.tempo_kv_element_offset(st.kv, which, j // Z, 0, j % Z, d)] = codes[j, d]
        pool.copy_(torch.from_numpy(raw))
    k, v = st.gather(0, rows)
    np.testing.assert_array_equal(np64(k)[0, :, 0], values)
    np.testing.assert_array_equal(np64(v)[0, :, 0], values)


@pytest.mark.parametrize("D,Z,B,t,count,ragged", [(128, 64, 3, 0, 1, False), (128, 32, 2, 5, 40, False), (64, 64, 2, 31, 66, False),
                                                  (128, 256, 2, 13, 300, False), (64, 32, 3, 40, 3, True), (128, 64, 3, 70, 100, True),
                                                  (64, 256, 1, 0, 513, False), (128, 32, 1, 63, 1, False), (128, 64, 2, 32, 64, False)])
def test_written_rows_come_back_and_others_stay(D, Z, B, t, count, ragged):
    Hkv = 3
    st = make_store(2, B, 2 * Hkv, Hkv, D, Z, t + count - 1)
    K, V = normal(7, 1, (B, count, Hkv, D)), normal(7, 2, (B, count, Hkv, D)) * 100
    K[0, 0, 0, 3], V[0, 0, 0, 5], K[-1, -1, -1] = np.inf, np.nan, 0.0
    first = synth.integers(4, 1, B, 0, t) if ragged else np.full(B, t)
    tps = torch.from_numpy(first.astype(np.int32)).to(DEV) if ragged else None
    st.append_block(bf16(K), bf16(V), t, count, tps)
    total = st.max_blocks_per_seq * Z
    k, v = st.gather(0, total)
    for got, x in ((k, K), (v, V)):
        for b in range(B):
            np.testing.assert_array_equal(np64(got)[b, first[b]:first[b] + count], held(np64(bf16(x[b]))))
    # every other byte still holds what it held
    own = np.zeros(st.k_pool.numel(), dtype=bool)
    table = st.block_table.cpu().numpy()
    for which, pool in ((0, st.k_pool), (1, st.v_pool)):
        own[:] = False
        codes = st.num_blocks * Hkv * Z * D
        for b in range(B):
            for j in range(first[b], first[b] + count):
                for h in range(Hkv):
                    at = [T.tempo_kv_element_offset(st.kv, which, int(table[b, j // Z]), h, j % Z, d) for d in (0, D - 1)]
                    assert max(at) < codes
                    own[T.tempo_kv_scale_offset(st.kv, which, int(table[b, j // Z]), h, j % Z)] = True
        left = pool.cpu().numpy() == 255
        assert left[codes:][~own[codes:]].all()
        assert (~left[:codes]).sum() <= B * count * Hkv * D


@pytest.mark.parametrize("t", [0, 1, 31, 40, 100])
@pytest.mark.parametrize("count", [128, 127, 97, 64])
def test_calls_that_fill_a_ring(t, count):
    """From any step on, the last group's slots among the first group's."""
    B, Hkv, D, Z, ring = 2, 2, 64, 64, 2
    st = make_store(9, B, Hkv, Hkv, D, Z, 0, ring)
    K, V = normal(9, 1, (B, count, Hkv, D)), normal(9, 2, (B, count, Hkv, D))
    st.append_block(bf16(K), bf16(V), t, count)
    k, v = st.gather(t, count)
    np.testing.assert_array_equal(np64(k), held(K))
    np.testing.assert_array_equal(np64(v), held(V))


@pytest.mark.parametrize("D,Z", [(64, 32), (128, 256)])
def test_offsets_beyond_32_bits(D, Z):
    """The last blocks of pools of more than 2^32 bytes."""
    Hq, Hkv, B, t = 6, 2, 1, 700
    blocks = (1 << 32) // (Hkv * Z * D) + 40
    pools = [torch.empty(blocks * Hkv * Z * (D + 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    table = torch.arange(blocks - 1, blocks - 1 - (t // Z + 1), -1, dtype=torch.int32).reshape(1, -1)
    st = BlockStore(B, Hq, Hkv, D, Z, t, E4M3, device=DEV, num_blocks=blocks, block_table=table, pools=pools)
    q, K, V = normal(10, 1, (B, Hq, D)), normal(10, 2, (B, t + 1, Hkv, D)), normal(10, 3, (B, t + 1, Hkv, D))
    st.append_block(bf16(K[:, :t]), bf16(V[:, :t]), 0, t)
    out = st.step_causal(bf16(q), bf16(K[:, t]), bf16(V[:, t]), st.new_out(), t)
    k, v = st.gather(0, t + 1)
    np.testing.assert_array_equal(np64(k), held(K))
    np.testing.assert_array_equal(np64(v), held(V))
    assert_attention(out, q, held(K), held(V), t, 0, st.scale, "far blocks")


@pytest.mark.parametrize("ring,Z,start", [(2, 32, 100), (4, 64, 1000)])
def test_ring_stores(ring, Z, start):
    B, Hq, Hkv, D = 2, 4, 2, 128
    steps, window = ring * Z, ring * Z - Z + 1
    st = make_store(3, B, Hq, Hkv, D, Z, 0, ring)
    q, K, V = normal(5, 1, (B, Hq, D)), normal(5, 2, (B, start + steps, Hkv, D)), normal(5, 3, (B, start + steps, Hkv, D))
    for t0 in range(0, start, steps):
        n = min(steps, start - t0)
        st.append_block(bf16(K[:, t0:t0 + n]), bf16(V[:, t0:t0 + n]), t0, n)
    out, t = st.new_out(), start - 1
    st.attend_window(bf16(q), out, t, window)
    assert_attention(out, q, held(K), held(V), t, window, st.scale, "ring")


@pytest.mark.parametrize("D,count", [(64, 1), (128, 1), (128, 70), (64, 33)])
def test_rotary_rows_are_rounded_to_bf16_and_then_quantised(D, count):
    """The store holds what appending the rotated rows (which are bf16) would have left, bit for bit."""
    B, Hkv, Z, t = 2, 2, 64, 37
    cos, sin = (torch.from_numpy(x.astype(np.float32)).to(DEV) for x in oracle.rope_table(t + count, D, 500000.0))
    a, c = (make_store(6, B, 2 * Hkv, Hkv, D, Z, t + count - 1) for _ in range(2))
    plain = BlockStore(B, 2 * Hkv, Hkv, D, Z, t + count - 1, T.TEMPO_BF16, device=DEV)
    K, V = bf16(normal(8, 1, (B, count, Hkv, D))), bf16(normal(8, 2, (B, count, Hkv, D)))
    for st in (a, plain):
        st.set_rope(cos, sin)
        st.rope_append_block(K, V, t, count)
    turned, _ = plain.gather(t, count)
    c.append_block(turned, V, t, count)
    assert torch.equal(a.k_pool, c.k_pool) and torch.equal(a.v_pool, c.v_pool)
    if count == 1:
        a.k_pool.fill_(255), a.v_pool.fill_(255)
        a.rope_append(K[:, 0].contiguous(), V[:, 0].contiguous(), t)
        assert torch.equal(a.k_pool, c.k_pool) and torch.equal(a.v_pool, c.v_pool)


# ---- attention --------------------------------------------------------------------------------------

CASES = [  # Hq, Hkv, D, Z, B, t, window, ragged, queries
    (6, 2, 128, 64, 2, 0, 0, False, 1), (6, 2, 128, 32, 3, 31, 0, False, 1), (8, 2, 64, 64, 2, 32, 0, False, 1),
    (24, 8, 128, 256, 2, 700, 0, False, 1), (24, 8, 128, 64, 5, 2049, 0, True, 1), (8, 8, 64, 32, 3, 500, 77, False, 1),
    (32, 4, 128, 64, 3, 900, 300, True, 1), (16, 1, 128, 64, 1, 5000, 0, False, 1), (17, 1, 64, 64, 2, 333, 0, False, 1),
    (128, 1, 128, 32, 1, 450, 100, False, 1), (80, 2, 64, 64, 2, 260, 0, True, 1),
    (6, 2, 128, 64, 2, 100, 0, False, 5), (6, 2, 64, 32, 2, 29, 10, False, 4), (24, 8, 128, 256, 2, 600, 0, True, 5),
    (4, 4, 128, 64, 2, 0, 0, False, 16), (6, 2, 128, 64, 2, 37, 0, False, 40), (12, 3, 64, 64, 1, 200, 50, True, 32),
    (4, 2, 128, 64, 1, 9000, 0, False, 1), (8, 2, 64, 64, 70, 40, 0, True, 1), (2, 2, 128, 64, 200, 300, 0, False, 1),
]


def filled(seed, Hq, Hkv, D, Z, B, t, window, ragged, queries):
    """A store that holds steps 0 .. t+queries-1 (of every sequence up to its own step) and nothing else."""
    n = t + queries
    q, K, V = normal(seed, 1, (B, queries, Hq, D)), normal(seed, 2, (B, n, Hkv, D)), normal(seed, 3, (B, n, Hkv, D))
    st = make_store(seed, B, Hq, Hkv, D, Z, n - 1)
    first = synth.integers(seed, 4, B, 0, t) if ragged else np.full(B, t)
    if ragged:
        first[0] = 0
    tps = torch.from_numpy(first.astype(np.int32)).to(DEV) if ragged else None
    if ragged:
        for b in range(B):
            one = T.make_kv(st.k_pool, st.v_pool, st.block_table[b], st.num_blocks, st.max_blocks_per_seq, Z, Hkv, D, E4M3)
            m = int(first[b]) + queries
            T.tempo_kv_append_block(one, bf16(K[b, :m]), bf16(V[b, :m]), 1, 0, None, m)
    else:
        st.append_block(bf16(K), bf16(V), 0, n)
    return st, q, held(K), held(V), first, tps


@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,window,ragged,queries", CASES)
def test_attention(Hq, Hkv, D, Z, B, t, window, ragged, queries):
    st, q, K, V, first, tps = filled(11, Hq, Hkv, D, Z, B, t, window, ragged, queries)
    if queries == 1:
        out = st.new_out()
        if window:
            st.attend_window(bf16(q[:, 0]), out, t, window, tps)
        else:
            st.attend_causal(bf16(q[:, 0]), out, t, tps)
        assert_attention(out, q[:, 0], K, V, first, window, st.scale, "step")
        return
    out = torch.empty((B, queries, Hq, D), dtype=torch.bfloat16, device=DEV)
    st.attend_block(bf16(q), out, t, queries, window, tps)
    for c in range(queries):
        assert_attention(out[:, c], q[:, c], K, V, first + c, window, st.scale, f"step {c}")


@pytest.mark.parametrize("tps,waves", [(32, 1), (64, 2), (128, 4), (256, 8), (1024, 8)])
@pytest.mark.parametrize("window", [0, 130])
def test_plans(tps, waves, window):
    Hq, Hkv, D, Z, B, t = 6, 2, 128, 64, 2, 611
    st, q, K, V, first, _ = filled(12, Hq, Hkv, D, Z, B, t, 0, False, 1)
    plan = T.tempo_plan(tps, t // tps + 1, waves)
    out = st.attend_with_plan(bf16(q[:, 0]), st.new_out(), t, plan, window)
    assert_attention(out, q[:, 0], K, V, first, window, st.scale, f"splits of {tps}")


@pytest.mark.parametrize("Hq,Hkv,D,B,t,ragged,window", [(24, 8, 128, 1, 299, False, 0), (8, 2, 64, 3, 64, True, 0), (40, 2, 128, 2, 95, False, 50),
                                                        (16, 16, 64, 40, 100, False, 0)])
def test_fused_steps_are_the_write_and_the_attention(Hq, Hkv, D, B, t, ragged, window):
    Z = 64
    a, q, K, V, first, tps = filled(13, Hq, Hkv, D, Z, B, t, window, ragged, 1)
    b, *_ = filled(13, Hq, Hkv, D, Z, B, t, window, ragged, 1)
    c, *_ = filled(13, Hq, Hkv, D, Z, B, t, window, ragged, 1)
    k, v = bf16(normal(14, 1, (B, Hkv, D))), bf16(normal(14, 2, (B, Hkv, D)))
    qd, one, two = bf16(q[:, 0]), a.new_out(), a.new_out()
    a.append(k, v, t, tps)
    if window:
        a.attend_window(qd, one, t, window, tps)
        b.step_window(qd, k, v, two, t, window, tps)
    else:
        a.attend_causal(qd, one, t, tps)
        b.step_causal(qd, k, v, two, t, tps)
    rows = np.arange(B)
    K[rows, first], V[rows, first] = held(np64(k)), held(np64(v))
    assert_attention(two, q[:, 0], K, V, first, window, a.scale, "fused step")
    assert_attention(one, q[:, 0], K, V, first, window, a.scale, "write, attend")
    assert torch.equal(a.k_pool, b.k_pool) and torch.equal(a.v_pool, b.v_pool)
    if not window:
        three = c.step_causal_noalloc(qd, k, v, a.new_out(), t, tps)
        assert torch.equal(three, two) and torch.equal(a.k_pool, c.k_pool) and torch.equal(a.v_pool, c.v_pool)


@pytest.mark.parametrize("D", [64, 128])
def test_unusual_rows_are_held_the_same_whichever_call_writes_them(D):
    """NaN, infinities, the largest values, zeros and rows of very different sizes, side by side in the heads of one step."""
    Hkv, B, Z, t = 8, 2, 32, 95                       # (step 95 completes its block)
    big = 3.3895313892515355e38                       # the largest bf16
    k = normal(61, 1, (B, Hkv, D))
    k[0, 1, 5], k[0, 2, D - 1], k[0, 3, 0], k[0, 4], k[0, 5] = np.nan, np.inf, -np.inf, 0.0, -big
    k[1, 0], k[1, 1, 7], k[1, 2], k[1, 3, 3], k[1, 4] = np.nan, big, k[1, 2] * 2.0 ** -125, 2.0 ** -133, np.inf
    k[1, 5, 1], k[1, 5, 2] = np.nan, big
    v = k[::-1, ::-1].copy()
    k, v, q = bf16(k), bf16(v), bf16(normal(61, 2, (B, Hkv, D)))
    before = bf16(normal(61, 3, (B, t, Hkv, D)))

    def written(call):
        st = make_store(61, B, Hkv, Hkv, D, Z, t)
        st.append_block(before, before, 0, t)
        call(st)
        return st.k_pool, st.v_pool

    pools = [written(lambda st: st.append(k, v, t)), written(lambda st: st.step_causal(q, k, v, st.new_out(), t)),
             written(lambda st: st.step_window(q, k, v, st.new_out(), t, 40)),
             written(lambda st: st.step_selected(st.new_bounds(), q, k, v, st.new_out(), t, 3)),
             written(lambda st: st.prefill_attend(q[:, None].contiguous(), k[:, None].contiguous(), v[:, None].contiguous(), st.new_out()[:, None].contiguous(), t, 1))]
    whole = make_store(61, B, Hkv, Hkv, D, Z, t)
    whole.append_block(torch.cat([before, k[:, None]], 1), torch.cat([before, v[:, None]], 1), 0, t + 1)  # by groups
    for kp, vp in pools:
        assert torch.equal(kp, whole.k_pool) and torch.equal(vp, whole.v_pool)
    got = whole.gather(t, 1)
    for x, row in zip(got, (k, v)):
        np.testing.assert_array_equal(np64(x)[:, 0], held(np64(row)))


@pytest.mark.parametrize("D,window,Hq,C", [(64, 0, 6, 4), (128, 0, 6, 4), (128, 40, 6, 4), (64, 0, 36, 7), (128, 33, 80, 3)])
def test_rotary_steps_and_blocks(D, window, Hq, C):
    Hkv, Z, B, t = 2, 64, 2, 150
    st, q, K, V, first, _ = filled(15, Hq, Hkv, D, Z, B, t, window, False, C)
    cos, sin = (torch.from_numpy(x.astype(np.float32)).to(DEV) for x in oracle.rope_table(t + C, D, 500000.0))
    st.set_rope(cos, sin)
    k, v = normal(16, 1, (B, Hkv, D)), normal(16, 2, (B, Hkv, D))
    turned_k, turned_q = st.rope_rotate(bf16(k), bf16(k), t), st.rope_rotate(bf16(q[:, 0]), bf16(q[:, 0]), t)
    out = st.rope_step(bf16(q[:, 0]), bf16(k), bf16(v), st.new_out(), t, window)
    K[:, t], V[:, t] = held(np64(turned_k)), held(v)
    assert_attention(out, np64(turned_q), K, V, first, window, st.scale, "rotary step")
    block = torch.empty((B, C, Hq, D), dtype=torch.bfloat16, device=DEV)
    st.attend_block(bf16(q), block, t, C, window, rope=True)
    for c in range(C):
        turned = st.rope_rotate(bf16(q[:, c]), bf16(q[:, c]), t + c)
        assert_attention(block[:, c], np64(turned), K, V, first + c, window, st.scale, f"rotary block, step {c}")


# ---- prompts ----------------------------------------------------------------------------------------

PROMPTS = [  # Hq, Hkv, D, Z, B, t, count, window, ring, rope, counts
    (6, 2, 128, 64, 2, 0, 1, 0, 0, False, False), (6, 2, 128, 64, 2, 0, 42, 0, 0, False, False), (6, 2, 128, 64, 2, 0, 43, 0, 0, False, False),
    (8, 2, 64, 32, 2, 37, 100, 0, 0, False, False), (24, 8, 128, 256, 2, 0, 300, 0, 0, False, False), (6, 2, 128, 64, 3, 0, 200, 0, 0, False, True),
    (6, 2, 128, 64, 3, 70, 20, 0, 0, False, True), (6, 2, 64, 64, 2, 50, 150, 0, 0, True, False), (6, 2, 128, 64, 2, 3, 20, 0, 0, True, False),
    (4, 2, 128, 32, 2, 500, 90, 33, 0, False, False), (4, 2, 128, 32, 2, 500, 90, 200, 0, True, True), (80, 1, 64, 64, 1, 20, 5, 0, 0, False, False),
    (6, 2, 128, 64, 2, 300, 250, 100, 4, False, False), (8, 8, 64, 32, 1, 77, 600, 40, 8, False, False), (6, 2, 128, 64, 1, 0, 30, 64, 2, False, False),
    (100, 1, 128, 64, 2, 0, 40, 0, 0, False, False),
]


@pytest.mark.parametrize("over_rows", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,count,window,ring,rope,counts", PROMPTS)
def test_prompts(Hq, Hkv, D, Z, B, t, count, window, ring, rope, counts, over_rows):
    """Every step of a prompt against the oracle over what the store holds after it; with over_rows, the answers lie over
    the prompt's own rows."""
    n = t + count
    q, K, V = normal(51, 1, (B, count, Hq, D)), normal(51, 2, (B, n, Hkv, D)), normal(51, 3, (B, n, Hkv, D))
    st = make_store(51, B, Hq, Hkv, D, Z, n - 1, ring)
    slots = ring * Z if ring else n
    for t0 in range(max(0, t - slots) // 32 * 32 if ring else 0, t, slots):
        m = min(slots, t - t0)
        st.append_block(bf16(K[:, t0:t0 + m]), bf16(V[:, t0:t0 + m]), t0, m)
    own = np.array([count, 0, count // 3])[:B] if counts else np.full(B, count)
    rows = torch.empty(2 * B * count * Hkv * D + B * count * Hq * D, dtype=torch.bfloat16, device=DEV)
    k_new, v_new = (rows[i * B * count * Hkv * D:(i + 1) * B * count * Hkv * D].view(B, count, Hkv, D) for i in (0, 1))
    k_new.copy_(bf16(K[:, t:])), v_new.copy_(bf16(V[:, t:]))
    out = (rows[:B * count * Hq * D] if over_rows else torch.empty(B * count * Hq * D, dtype=torch.bfloat16, device=DEV)).view(B, count, Hq, D)
    if rope:
        cos, sin = (torch.from_numpy(x.astype(np.float32)).to(DEV) for x in oracle.rope_table(n, D, 500000.0))
        st.set_rope(cos, sin)
        for c in range(count):
            q[:, c], K[:, t + c] = (np64(st.rope_rotate(bf16(x), bf16(x), t + c)) for x in (q[:, c], K[:, t + c]))
    raw_q = normal(51, 1, (B, count, Hq, D))
    before = out.clone()
    need = T.tempo_prefill_workspace_bytes(st.kv, B, Hq, n - 1 if not ring else slots + 128)
    if ring:
        need += 4 * rows.numel()
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    args = (B, Hq, t, count, torch.from_numpy(own.astype(np.int32)).to(DEV) if counts else None)
    if window:
        args += (window,)
    call = {(0, 0): T.tempo_prefill_causal, (1, 0): T.tempo_prefill_window, (0, 1): T.tempo_rope_prefill_causal, (1, 1): T.tempo_rope_prefill_window}
    lead = (st.kv, st.rope) if rope else (st.kv,)
    call[(int(window > 0), int(rope))](*lead, bf16(raw_q), k_new, v_new, out, *args, st.scale, ws, need)
    Kh, Vh = held(K), held(V)
    for c in sorted({0, 1, 2, 31, 32, 63, 64, count // 2, count - 2, count - 1}):
        live = [b for b in range(B) if 0 <= c < own[b]]
        if live:
            assert_attention(out[live, c], q[live, c], Kh[live], Vh[live], t + c, window, st.scale, f"step {c}")
    for b in range(B):
        if not over_rows:
            assert torch.equal(out[b, own[b]:].view(torch.int16), before[b, own[b]:].view(torch.int16))
        last = t + own[b]
        first = max(0, last - slots) if ring else 0
        if last > first:
            kg, vg = st.gather(first, last - first)
            np.testing.assert_array_equal(np64(kg)[b], Kh[b, first:last])
            np.testing.assert_array_equal(np64(vg)[b], Vh[b, first:last])


@pytest.mark.parametrize("Hq,Hkv,D,Z,B,count,window,counts", [(6, 2, 128, 64, 2, 150, 0, False), (6, 2, 64, 32, 3, 200, 0, True), (8, 2, 64, 256, 2, 301, 50, False)])
def test_rotary_prompts_from_the_first_step_on(Hq, Hkv, D, Z, B, count, window, counts):
    for over_rows in (False, True):
        test_prompts(Hq, Hkv, D, Z, B, 0, count, window, 0, True, counts, over_rows)


@pytest.mark.parametrize("Hq,Hkv,D,Z,t,count,window", [(6, 2, 128, 64, 0, 200, 0), (8, 2, 64, 32, 0, 333, 0), (6, 2, 128, 64, 0, 300, 77), (6, 2, 128, 32, 70, 150, 0),
                                                     (8, 8, 64, 64, 0, 33, 0)])
def test_prompts_do_not_depend_on_what_the_workspace_held(Hq, Hkv, D, Z, t, count, window):
    """Prompts of different lengths side by side; a workspace of zeros, of NaN, and what the calls before left."""
    own = np.array([count, 0, count // 3, 1, count - 1, 32])
    B = len(own)
    q, K, V = normal(57, 1, (B, count, Hq, D)), normal(57, 2, (B, t + count, Hkv, D)), normal(57, 3, (B, t + count, Hkv, D))
    answers = []
    ws = None
    for fill in (0, 255, None):
        st = make_store(57, B, Hq, Hkv, D, Z, t + count - 1)
        if t:
            st.append_block(bf16(K[:, :t]), bf16(V[:, :t]), 0, t)
        need = T.tempo_prefill_workspace_bytes(st.kv, B, Hq, t + count - 1)
        ws = torch.full((need,), fill, dtype=torch.uint8, device=DEV) if fill is not None else ws
        out = torch.zeros((B, count, Hq, D), dtype=torch.bfloat16, device=DEV)
        args = (B, Hq, t, count, ints(own)) + ((window,) if window else ())
        call = T.tempo_prefill_window if window else T.tempo_prefill_causal
        call(st.kv, bf16(q), bf16(K[:, t:]), bf16(V[:, t:]), out, *args, st.scale, ws, need)
        answers.append(out)
    assert all(torch.equal(a, answers[0]) for a in answers)
    Kh, Vh = held(K), held(V)
    for c in sorted({0, 31, 32, count // 3 - 1, count - 1}):
        live = [b for b in range(B) if c < own[b]]
        if live:
            assert_attention(answers[0][live, c], q[live, c], Kh[live], Vh[live], t + c, window, D ** -0.5, f"step {c}")
    for b in range(B):
        assert not answers[0][b, own[b]:].any()


@pytest.mark.parametrize("over_rows", [False, True])
@pytest.mark.parametrize("Hq,Hkv,D,Z,B,t,count,window,ring,rope,counts",
                         [(6, 2, 128, 64, 2, 2500, 60, 0, 0, False, False), (8, 2, 64, 32, 1, 3000, 64, 0, 0, True, False),
                          (32, 1, 128, 256, 1, 3700, 6, 0, 0, False, False), (6, 2, 128, 64, 2, 2000, 45, 600, 16, False, False),
                          (6, 2, 64, 64, 2, 1000, 43, 300, 0, True, False), (6, 2, 128, 64, 1, 1000, 130, 200, 8, False, False)])
def test_prompts_of_two_blocks_behind_a_history(Hq, Hkv, D, Z, B, t, count, window, ring, rope, counts, over_rows):
    test_prompts(Hq, Hkv, D, Z, B, t, count, window, ring, rope, counts, over_rows)


def test_nan_shows_where_it_is_seen_only():
    Hq, Hkv, D, Z, B, t, window = 6, 2, 128, 64, 2, 300, 100
    q, K, V = normal(17, 1, (B, Hq, D)), normal(17, 2, (B, t + 1, Hkv, D)), normal(17, 3, (B, t + 1, Hkv, D))
    K[0, 150, 0, 7], V[1, 250, 1, 9], K[1, :, 0, 0] = np.nan, np.inf, np.nan
    st = make_store(17, B, Hq, Hkv, D, Z, t)
    st.append_block(bf16(K), bf16(V), 0, t + 1)
    causal, windowed = np64(st.attend_causal(bf16(q), st.new_out(), t)), np64(st.attend_window(bf16(q), st.new_out(), t, window))
    assert np.isnan(causal[0, :3]).all() and np.isfinite(causal[0, 3:]).all()
    assert np.isfinite(windowed[0]).all()
    for got in (causal, windowed):
        assert np.isnan(got[1, :3]).all()                          # every key is NaN
        assert np.isnan(got[1, 3:, 9]).all() and np.isfinite(np.delete(got[1, 3:], 9, axis=-1)).all()


def test_far_from_one():
    """Rows of 2^100 and 2^-100: scales near both ends of the range, logits in reach through the scale argument."""
    Hq, Hkv, D, Z, B, t = 4, 2, 64, 32, 1, 90
    for power in (100, -100):
        q, K, V = normal(18, 1, (B, Hq, D)), normal(18, 2, (B, t + 1, Hkv, D)), normal(18, 3, (B, t + 1, Hkv, D)) * 2.0 ** power
        st = make_store(18, B, Hq, Hkv, D, Z, t)
        st.append_block(bf16(K), bf16(V), 0, t + 1)
        out = st.attend_causal(bf16(q), st.new_out(), t)
        assert_attention(out, q, held(K), held(V), t, 0, st.scale, f"values of 2^{power}")


@pytest.mark.parametrize("queries", [1, 30])
def test_values_at_the_end_of_the_range(queries):
    """Averages of values of up to 3e38 over 200 keys of nearly the same weight: sums of weights times values stay finite."""
    B, Hq, Hkv, D, Z, n = 2, 6, 2, 128, 64, 200
    q, K = normal(71, 1, (B, queries, Hq, D)) * 2.0 ** -6, normal(71, 2, (B, n, Hkv, D))
    V = np.abs(normal(71, 3, (B, n, Hkv, D)))
    V = np64(bf16(np.minimum(1 + V, 1.99) * 2.0 ** 127))
    st = make_store(71, B, Hq, Hkv, D, Z, n - 1)
    st.append_block(bf16(K), bf16(V), 0, n)
    out = torch.empty((B, queries, Hq, D), dtype=torch.bfloat16, device=DEV)
    t = n - queries
    st.attend_block(bf16(q), out, t, queries)
    for c in sorted({0, queries - 1}):
        assert_attention(out[:, c], q[:, c], held(K), held(V), t + c, 0, st.scale, f"step {c}")


def test_captured_and_replayed_and_on_another_stream():
    Hq, Hkv, D, Z, B, t = 24, 8, 128, 64, 2, 1500
    st, q, K, V, first, _ = filled(19, Hq, Hkv, D, Z, B, t, 0, False, 1)
    k, v, qd = bf16(K[:, t]), bf16(V[:, t]), bf16(q[:, 0])
    eager = st.step_causal(qd, k, v, st.new_out(), t).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = st.step_causal(qd, k, v, st.new_out(), t)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(eager, other)
    out = st.new_out()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st.step_causal(qd, k, v, out, t)
    for i in range(4):
        qd.copy_(bf16(normal(20 + i, 1, (B, Hq, D))))
        eager = st.step_causal(qd, k, v, st.new_out(), t).clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


@pytest.mark.parametrize("t,count,window", [(0, 200, 0), (300, 100, 0), (2500, 60, 0), (0, 300, 70)])
def test_prompts_captured_and_replayed(t, count, window):
    """Rows written and laid out at once; turned by a launch of their own; two blocks over the codes.  Other rows and queries on
    every replay, another prompt and its own eager run in between."""
    Hq, Hkv, D, Z, B = 6, 2, 128, 64, 2
    st, other = make_store(63, B, Hq, Hkv, D, Z, t + count - 1), make_store(64, B, Hq, Hkv, D, Z, t + count - 1)
    if t:
        before = bf16(normal(63, 1, (B, t, Hkv, D)))
        st.append_block(before, before, 0, t), other.append_block(before, before, 0, t)
    q, k, v = bf16(normal(63, 2, (B, count, Hq, D))), bf16(normal(63, 3, (B, count, Hkv, D))), bf16(normal(63, 4, (B, count, Hkv, D)))
    out, eager = torch.empty_like(q), torch.empty_like(q)
    st.prefill_attend(q, k, v, out, t, count, window)  # (the workspace is there before the capture)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        st.prefill_attend(q, k, v, out, t, count, window)
    for i in range(4):
        for x, which in ((q, 5), (k, 6), (v, 7)):
            x.copy_(bf16(normal(70 + i, which, x.shape)))
        other.prefill_attend(q, k, v, eager, t, count, window)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        assert all(torch.equal(a, b) for a, b in zip(st.gather(t, count), other.gather(t, count)))
