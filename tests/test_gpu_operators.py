"""Rotary positions with several axes, attention of packed sequences, keys and values in 8-bit pages and attention over them, through the
C ABI, against plain 64-bit definitions (operator_refs.py, where the tolerances are derived)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import operator_refs as ref  # noqa: E402

BF16_P = 2.0 ** -8                  # probabilities rounded to bf16 once


def _bd():
    from paper_2509_11628_amd import binding as bd
    return bd


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


# ---- rotary positions -------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,dims", [(128, (16, 56, 56)), (72, (32, 32)), (72, (24, 24, 24)), (64, (64,)), (64, (16, 16, 16, 16)), (16, (4, 4)), (30, (6, 10, 8)), (128, (64,))])
@pytest.mark.parametrize("halves", [False, True])
def test_rope(dtype, hd, dims, halves):
    """Both spectra, with and without norm, whole and partial rotation, grouped heads, far and negative positions, odd token counts."""
    bd = _bd()
    for i, (tokens, H, Hkv, joint, normed) in enumerate([(1, 1, 1, False, False), (7, 6, 2, True, True), (257, 5, 5, False, True), (40, 32, 8, True, False)]):
        dt = _dt(dtype)
        q, k = ref.randn((tokens, H, hd), dt, 1 + i), ref.randn((tokens, Hkv, hd), dt, 50 + i, 30.0)
        g = torch.Generator(device="cuda").manual_seed(i)
        pos = torch.randint(-50, 1000000, (tokens, len(dims)), generator=g, device="cuda", dtype=torch.int32)
        theta, scale = [10000.0, 500.0, 1.0e6, 3.0][:len(dims)], [1.0, 0.5, 0.25, 2.0][:len(dims)]
        norms = [1.0 + ref.randn((hd,), dt, 90 + j, 0.1) if normed else None for j in range(2)]
        rope = bd.make_rope(dims, theta, scale, bd.ROPE_HALVES if halves else bd.ROPE_ADJACENT, bd.ROPE_JOINT if joint else bd.ROPE_PER_AXIS)
        got = bd.rope_axes(rope, pos, q, k, norms[0], norms[1], eps=1e-5)
        for x, y, norm in zip((q, k), got, norms):
            ref.close(y, *ref.rope(x, pos, dims, theta, scale, halves, joint, norm, 1e-5), (tokens, H, joint, normed))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 8), (4, 4), (2, 2), (1, 1), (0, 1)])
def test_rope_strides_in_place_and_alone(dtype, pad, offset):
    """Views of any alignment give the bits of aligned ones, in place as well as not, q alone as well as with k; what lies between stays."""
    bd = _bd()
    dt = _dt(dtype)
    for hd, dims in ((64, (32, 32)), (72, (24, 24, 24)), (72, (32, 32)), (128, (16, 56, 56))):
        for pairing in (bd.ROPE_ADJACENT, bd.ROPE_HALVES):
            q, k, norm = ref.randn((33, 3, hd), dt, 1), ref.randn((33, 2, hd), dt, 2), 1.0 + ref.randn((hd,), dt, 3, 0.1)
            pos = torch.arange(33 * len(dims), device="cuda", dtype=torch.int32).view(33, len(dims))
            rope = bd.make_rope(dims, pairing=pairing)
            want = bd.rope_axes(rope, pos, q, k, norm, None)
            qs, ks = ref.strided(q, pad, offset), ref.strided(k, pad, offset)
            got = bd.rope_axes(rope, pos, qs, ks, norm, None)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            alone = bd.rope_axes(rope, pos, qs, q_norm=norm)
            assert torch.equal(alone, want[0])
            bd.rope_axes(rope, pos, qs, ks, norm, None, out=(qs, ks))
            assert torch.equal(qs, want[0]) and torch.equal(ks, want[1])
            if pad:
                rest = qs.as_strided((32, pad), (qs.stride(0), 1), qs.storage_offset() + 3 * hd)
                assert bool((rest == 3.0).all())


def test_rope_no_tokens_and_position_zero():
    bd = _bd()
    q = ref.randn((5, 4, 64), torch.float32, 1)
    rope = bd.make_rope((32, 32))
    assert torch.equal(bd.rope_axes(rope, torch.zeros((5, 2), dtype=torch.int32, device="cuda"), q), q)
    assert bd.rope_axes(rope, torch.zeros((0, 2), dtype=torch.int32, device="cuda"), q[:0]).shape == (0, 4, 64)


def test_rope_matches_tables_of_a_grid():
    """Positions of a (time, height, width) grid behind text at the origin give what cos / sin tables over the axes give."""
    bd = _bd()
    T, h, w, text, axes = 3, 5, 4, 7, (16, 24, 24)
    grid = torch.stack(torch.meshgrid(*(torch.arange(n) for n in (T, h, w)), indexing="ij"), -1).view(-1, 3)
    pos = torch.cat([torch.zeros((text, 3), dtype=torch.int64), grid]).to(device="cuda", dtype=torch.int32)
    q = ref.randn((len(pos), 2, 64), torch.float32, 3)
    got = bd.rope_axes(bd.make_rope(axes), pos, q)
    ref.close(got, *ref.rope(q, pos, axes, [10000.0] * 3, [1.0] * 3, False, False, None, 0.0))
    assert torch.equal(got[:text], q[:text])


# ---- packed attention ---------------------------------------------------------------------------------------


def _packed_check(bd, lens, H, Hkv, hd, dtype, causal, seed=0, scale=0.0, first=0, behind=3, pad=0, offset=0, spread=1.0):
    dt = _dt(dtype)
    total = first + sum(lens) + behind
    q, k, v = ref.randn((total, H, hd), dt, seed + 1, spread), ref.randn((total, Hkv, hd), dt, seed + 2), ref.randn((total, Hkv, hd), dt, seed + 3)
    starts = ref.starts_of(lens, first)
    out = torch.full((total, H, hd), 5.0, dtype=dt, device="cuda")
    if pad or offset:
        q, k, v, out = (ref.strided(x, pad, offset) for x in (q, k, v, out))
    got = bd.attention_packed(q, k, v, starts, causal=causal, scale=scale, out=out)
    at = first
    for n in lens:
        sees = torch.ones((n, n), dtype=torch.bool, device="cuda")
        if causal:
            sees = sees.tril()
        # the fp32 kernel keeps probabilities in fp32; the tolerance allows for both
        p_step = BF16_P if dtype == "bf16" else 0.0
        ref.close(got[at:at + n], *ref.attention(q[at:at + n], k[at:at + n], v[at:at + n], sees, scale or 1.0 / math.sqrt(hd), p_step, dt), (lens, n, H, hd, causal))
        at += n
    assert bool((got[:first] == 5.0).all()) and bool((got[at:] == 5.0).all())
    return q, k, v, starts, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [16, 32, 64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_packed(dtype, hd, causal):
    """Lengths around every tile size, empty sequences, grouped heads, rows ahead of the first and behind the last sequence."""
    bd = _bd()
    _packed_check(bd, [1], 1, 1, hd, dtype, causal)
    _packed_check(bd, [0, 1, 2, 15, 16, 17, 0, 31, 32, 33, 63, 64, 65, 0], 4, 2, hd, dtype, causal, first=5)
    _packed_check(bd, [127, 128, 129, 191, 193, 255, 256, 257, 300], 3, 1, hd, dtype, causal)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 72), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_packed_long_and_many(dtype, hd, causal):
    bd = _bd()
    _packed_check(bd, [1500, 3, 700], 8, 2, hd, dtype, causal, seed=5)
    rng = np.random.default_rng(1)
    _packed_check(bd, rng.integers(0, 9, 300).tolist(), 2, 2, hd, dtype, causal, seed=6)       # more sequences than a wave has lanes
    _packed_check(bd, [200, 500], 6, 6, hd, dtype, causal, seed=7, scale=0.5, spread=4.0)      # peaked, another scale


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 72), ("f32", 72), ("f32", 128)])
@pytest.mark.parametrize("pad,offset", [(8, 8), (4, 4), (1, 0), (0, 1)])
def test_packed_strides(dtype, hd, pad, offset):
    bd = _bd()
    _packed_check(bd, [70, 130, 1], 4, 2, hd, dtype, True, seed=9, pad=pad, offset=offset)


def test_packed_views_of_one_layer():
    """q, k and v as views of one layer's output [tokens, (H + 2 Hkv) hd]."""
    bd = _bd()
    H, Hkv, hd, lens = 8, 2, 128, [100, 29]
    qkv = ref.randn((129, (H + 2 * Hkv) * hd), torch.bfloat16, 3)
    q, k, v = qkv[:, :H * hd].view(129, H, hd), qkv[:, H * hd:(H + Hkv) * hd].view(129, Hkv, hd), qkv[:, (H + Hkv) * hd:].view(129, Hkv, hd)
    got = bd.attention_packed(q, k, v, ref.starts_of(lens))
    assert torch.equal(got, bd.attention_packed(q.contiguous(), k.contiguous(), v.contiguous(), ref.starts_of(lens)))


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("bf16", 72), ("bf16", 64), ("f32", 64), ("f32", 72), ("bf16", 32)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_packed_hidden_values_have_no_part(dtype, hd, bad):
    """What lies in other sequences, or behind a causal token, is no number: results stay those without it."""
    bd = _bd()
    lens, H, Hkv, at = [90, 200, 50], 4, 2, 90 + 77
    total = sum(lens)
    dt = _dt(dtype)
    q, k, v = ref.randn((total, H, hd), dt, 1), ref.randn((total, Hkv, hd), dt, 2), ref.randn((total, Hkv, hd), dt, 3)
    starts = ref.starts_of(lens)
    for causal in (False, True):
        clean = bd.attention_packed(q, k, v, starts, causal=causal)
        for x in (k, v):
            old = x[at].clone()
            x[at] = bad
            got = bd.attention_packed(q, k, v, starts, causal=causal)
            x[at] = old
            keep = torch.ones(total, dtype=torch.bool, device="cuda")
            keep[at if causal else 90:290] = False
            assert torch.equal(got[keep], clean[keep]), (causal, x is v)
            seen = got[at:290].float()
            if x is v:
                want = math.nan if math.isnan(bad) else bad
                assert bool((seen.isnan() if math.isnan(want) else seen == want).all())
            elif math.isnan(bad):
                assert bool(seen.isnan().all())


def test_packed_offsets_that_are_none():
    """Offsets outside the buffer or falling: nothing outside is touched, the call ends."""
    bd = _bd()
    q, k, v = (ref.randn((100, 2, 64), torch.bfloat16, i) for i in range(3))
    for cu in ([0, 50, 1000], [-7, 20, 100], [0, 80, 30, 100], [100, 100], [2000, 3000]):
        out = bd.attention_packed(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), out=torch.zeros_like(q))
        torch.cuda.synchronize()
        assert bool(out.isfinite().all())


def test_packed_matches_plain_attention_of_equal_lengths():
    """Equal lengths, as many key heads as heads, no mask: the packed call and the plain one agree to their rounding."""
    bd = _bd()
    rows, T, H, hd = 3, 320, 6, 64
    qkv = ref.randn((rows, T, 3 * H * hd), torch.bfloat16, 1)
    flat = qkv.view(rows * T, 3, H, hd)
    got = bd.attention_packed(flat[:, 0], flat[:, 1], flat[:, 2], ref.starts_of([T] * rows))
    want = bd.attention(qkv, H).view(rows * T, H, hd).double()
    # each is within (one rounding of P) x sum p |v| + one of the result; sum p |v| <= max |v|
    assert float((got.double() - want).abs().max()) <= 2 * 2.0 ** -8 * float(flat[:, 2].abs().max()) * 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_beyond_32_bits(dtype):
    """Tokens whose elements lie more than 2^32 bytes behind the first, in attention and in the rotation."""
    bd = _bd()
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    total, H, hd, lens = 290_000, 64, 128, [130, 70]
    n = sum(lens)
    q, k, v = (torch.empty((total, H, hd), dtype=dt, device="cuda") for _ in range(3))
    for i, x in enumerate((q, k, v)):
        x[-n:] = ref.randn((n, H, hd), dt, i)
    assert (total - n) * H * hd * q.element_size() > 2 ** 32
    for causal in (False, True):
        got = bd.attention_packed(q, k, v, ref.starts_of(lens, total - n), causal=causal)
        at = total - n
        for m in lens:
            sees = torch.ones((m, m), dtype=torch.bool, device="cuda")
            x = [t[at:at + m] for t in (q, k, v)]
            ref.close(got[at:at + m], *ref.attention(*x, sees.tril() if causal else sees, hd ** -0.5, BF16_P if dtype == "bf16" else 0.0, dt))
            at += m
    rope, pos = bd.make_rope((64, 64)), torch.arange(2 * total, dtype=torch.int32, device="cuda").view(total, 2)
    q[:-n] = 1.0
    want = bd.rope_axes(rope, pos[-n:].clone(), q[-n:].clone())
    bd.rope_axes(rope, pos, q, out=q)
    assert torch.equal(q[-n:], want)


# ---- the cache ----------------------------------------------------------------------------------------------


def _new_cache(bd, pages, heads, hd, seed=0):
    """Pages full of bytes that mean nothing (NaN among them), so that what is not held must not be looked at."""
    c = bd.KVCache.empty(pages, heads, hd)
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.k.random_(0, 256, generator=g)
    c.v.random_(0, 256, generator=g)
    c.k_scale.fill_(2.0 ** 60)
    c.v_scale.fill_(2.0 ** 60)
    return c


def _tables(pages, counts, width, seed=0):
    order = np.random.default_rng(seed).permutation(pages)
    t, at = np.full((len(counts), width), -1, np.int32), 0
    for s, n in enumerate(counts):
        t[s, :n] = order[at:at + n]
        at += n
    return t


def _dev(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _same_cache(dev, want):
    got = ref.Cache(dev)
    for a, b, name in zip(got.s + got.b, want.s + want.b, ("k scale", "v scale", "k", "v")):
        same = a == b if a.dtype != np.uint8 else (a == b) | (((a & 127) == 127) & ((b & 127) == 127))
        assert same.all(), (name, int((~same).sum()), np.argwhere(~same)[:4].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [16, 32, 64, 72, 128])
def test_store_and_load(dtype, hd):
    """Three rounds of growth: bytes and scales to the bit, also of pages that grow (scales rise, old tokens are rounded again), pages that
    nothing wrote, and the values read back."""
    bd = _bd()
    dt, heads = _dt(dtype), 3
    cache = _new_cache(bd, 40, heads, hd)
    want = ref.Cache(cache)
    table = _tables(40, [6, 7, 1, 9], 9)
    past = np.zeros(4, np.int64)
    for turn, lens in enumerate([(1, 130, 0, 63), (64, 70, 5, 1), (200, 1, 59, 300)]):
        lens = np.array(lens)
        total = int(lens.sum()) + 2
        k, v = ref.randn((total, heads, hd), dt, 10 + turn, (0.01, 1.0, 37.0)[turn]), ref.randn((total, heads, hd), dt, 20 + turn, (300.0, 1e-6, 1.0)[turn])
        starts = ref.starts_of(lens.tolist(), 1)
        bd.kv_store(cache, _dev(table), _dev(past), k, v, starts)
        want.store(table.tolist(), past.tolist(), k, v, starts.tolist(), lens.tolist())
        _same_cache(cache, want)
        past += lens
    out = [torch.full((int(past.sum()) + 2, heads, hd), 9.0, dtype=dt, device="cuda") for _ in range(2)]
    first = np.array([3, 64, 0, 65])
    lens = past - first
    bd.kv_load(cache, _dev(table), _dev(first), ref.starts_of(lens.tolist(), 1), out[0].shape[0], dt, out=out)
    for which in range(2):
        at = 1
        for s, n in enumerate(lens):
            vals, held = want.values(which, table[s], int(past[s]))
            assert bool(held.all()) and torch.equal(out[which][at:at + n].double(), vals[first[s]:])
            at += n
        assert bool((out[which][:1] == 9.0).all()) and bool((out[which][at:] == 9.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_values_at_the_borders(dtype):
    """Zeros, infinities, NaN, the smallest and largest numbers, ties, and maxima at and next to 448 x 2^e."""
    bd = _bd()
    dt, hd = _dt(dtype), 64
    big = float(torch.finfo(dt).max)
    rows = [[0.0], [math.inf, 1.0], [-math.inf, math.nan, 3.0], [big, -big, 1.0], [1e-38, -1e-38], [448.0], [449.0 if dt == torch.float32 else 450.0], [math.nan],
            [1.0625, 1.1875, -1.0625, 17.0, 19.0, 448.0], [2.0 ** -9, 1.5 * 2.0 ** -9, 2.5 * 2.0 ** -9, 2.0 ** -10, 448.0], [math.inf], [0.0, -0.0, 448.0 * 2.0 ** -100], [1.0]]
    if dt == torch.float32:
        rows += [[np.nextafter(np.float32(448.0), np.float32(500.0))], [1e-45], [448.0 * 2.0 ** 119]]
    cache, n = _new_cache(bd, len(rows), 1, hd), len(rows)
    want = ref.Cache(cache)
    x = torch.zeros((n * 2, 1, hd), dtype=dt, device="cuda")
    for i, r in enumerate(rows):
        x[2 * i, 0, :len(r)] = torch.tensor(r, dtype=torch.float64).to(dt).cuda()
        x[2 * i + 1, 0, 5:5 + len(r)] = -x[2 * i, 0, :len(r)]
    table, past, starts = np.arange(n)[:, None], [0] * n, ref.starts_of([2] * n)
    bd.kv_store(cache, _dev(table), _dev(past), x, x.flip(2).contiguous(), starts)
    want.store(table.tolist(), past, x, x.flip(2), starts.tolist(), [2] * n)
    _same_cache(cache, want)
    # the same tokens once more behind themselves: pages that grow
    bd.kv_store(cache, _dev(table), _dev([2] * n), x, x, starts)
    want.store(table.tolist(), [2] * n, x, x, starts.tolist(), [2] * n)
    _same_cache(cache, want)
    k, v = bd.kv_load(cache, _dev(table), _dev(past), ref.starts_of([4] * n), 4 * n, dt)
    for which, got in enumerate((k, v)):
        for i in range(n):
            vals, _ = want.values(which, table[i], 4)
            assert torch.equal(got[4 * i:4 * i + 4].double().nan_to_num(nan=12345.0), vals.to(dt).double().nan_to_num(nan=12345.0))


def test_pages_that_are_none():
    """Page numbers outside the cache, tokens behind the table's end, runs that begin below 0: nothing is stored, loads give zeros
    (rows of a run below 0 stay), attention leaves them out."""
    bd = _bd()
    heads, hd = 2, 64
    cache = _new_cache(bd, 4, heads, hd)
    want = ref.Cache(cache)
    table = np.array([[2, -1, 99, 1], [4, 0, -5, 3]])
    lens = [300, 256]
    k, v = ref.randn((556, heads, hd), torch.bfloat16, 1), ref.randn((556, heads, hd), torch.bfloat16, 2)
    starts = ref.starts_of(lens)
    bd.kv_store(cache, _dev(table), _dev([0, 0]), k, v, starts)
    want.store(table.tolist(), [0, 0], k, v, starts.tolist(), lens)
    _same_cache(cache, want)
    bd.kv_store(cache, _dev(table), _dev([-3, -64]), k, v, starts)
    _same_cache(cache, want)
    got = bd.kv_load(cache, _dev(table), _dev([0, 0]), starts, 556, torch.bfloat16)
    for which in range(2):
        for s, at in ((0, 0), (1, 300)):
            vals, held = want.values(which, table[s], lens[s])
            assert torch.equal(got[which][at:at + lens[s]].double(), vals) and not bool(held.all())
    q = ref.randn((2, 4, hd), torch.bfloat16, 3)
    out = bd.attention_cached(q, ref.starts_of([1, 1]), cache, _dev(table), _dev([300, 256]), causal=True)
    for s in range(2):
        (kk, held), (vv, _) = want.values(0, table[s], lens[s]), want.values(1, table[s], lens[s])
        ref.close(out[s:s + 1], *ref.attention(q[s:s + 1], kk, vv, held[None], 0.125, BF16_P, torch.bfloat16))
    nothing = bd.attention_cached(q, ref.starts_of([1, 1]), cache, _dev(np.full((2, 4), -1)), _dev([300, 256]))
    assert bool((nothing == 0).all())


@pytest.mark.parametrize("pad,offset", [(8, 8), (4, 4), (1, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("hd", [64, 72])
def test_cache_strides(pad, offset, hd):
    bd = _bd()
    heads, lens = 3, [70, 1, 64]
    table = _tables(8, [2, 1, 2], 2)
    k, v = ref.randn((135, heads, hd), torch.bfloat16, 1), ref.randn((135, heads, hd), torch.bfloat16, 2)
    a, b = _new_cache(bd, 8, heads, hd), _new_cache(bd, 8, heads, hd)
    past, starts = _dev([5, 0, 3]), ref.starts_of(lens)
    a.k.zero_(); b.k.zero_(); a.v.zero_(); b.v.zero_()
    bd.kv_store(a, _dev(table), past, k, v, starts)
    bd.kv_store(b, _dev(table), past, ref.strided(k, pad, offset), ref.strided(v, pad, offset), starts)
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v) and torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)
    want = bd.kv_load(a, _dev(table), past, starts, 135, torch.bfloat16)
    out = [ref.strided(torch.zeros_like(k), pad, offset) for _ in range(2)]
    bd.kv_load(a, _dev(table), past, starts, 135, torch.bfloat16, out=out)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    q = ref.randn((5, 6, hd), torch.bfloat16, 4)
    cu, held = ref.starts_of([2, 1, 2]), _dev([75, 1, 67])
    plain = bd.attention_cached(q, cu, a, _dev(table), held)
    strided = bd.attention_cached(ref.strided(q, pad, offset), cu, a, _dev(table), held, out=ref.strided(torch.zeros_like(q), pad, offset))
    assert torch.equal(plain, strided)


# ---- attention over the cache -----------------------------------------------------------------------------------


def _fill(bd, lens, heads, hd, seed=0, spread=1.0):
    """A cache of sequences of these lengths behind which lie bytes that mean nothing, with its table and its 64-bit twin."""
    counts = [(n + 63) // 64 for n in lens]
    pages = sum(counts) + 3
    cache = _new_cache(bd, pages, heads, hd, seed)
    table = _tables(pages, counts, max(counts) + 1, seed)
    total = sum(lens)
    k, v = ref.randn((total, heads, hd), torch.bfloat16, seed + 1, spread), ref.randn((total, heads, hd), torch.bfloat16, seed + 2)
    if total:
        bd.kv_store(cache, _dev(table), _dev([0] * len(lens)), k, v, ref.starts_of(lens))
    # behind the last token of a page: NaN again, as of a sequence that was longer once
    for s, n in enumerate(lens):
        if n % 64:
            cache.k[int(table[s, n // 64]), :, n % 64:] = 0x7F
            cache.v[int(table[s, n // 64])][:, :, torch.tensor(ref.PLACE[n % 64:], device="cuda")] = 0xFF
    return cache, table, ref.Cache(cache)


def _cached_check(bd, new, lens, H, Hkv, hd, causal, seed=0, scale=0.0, max_len=None, first=2, behind=2, spread=1.0):
    cache, table, twin = _fill(bd, lens, Hkv, hd, seed, spread)
    total = first + sum(new) + behind
    q = ref.randn((total, H, hd), torch.bfloat16, seed + 7)
    out = torch.full((total, H, hd), 5.0, dtype=torch.bfloat16, device="cuda")
    got = bd.attention_cached(q, ref.starts_of(new, first), cache, _dev(table), _dev(lens), causal=causal, scale=scale, max_len=max_len, out=out)
    at = first
    for s, (a, n) in enumerate(zip(new, lens)):
        (k, held), (v, _) = twin.values(0, table[s], n), twin.values(1, table[s], n)
        sees = held[None].expand(a, n)
        if max_len is not None:
            sees = sees & (torch.arange(n, device="cuda") < max_len)[None]
        if causal:
            m = n if max_len is None else min(n, max_len)
            sees = sees & (torch.arange(n, device="cuda")[None] <= m - a + torch.arange(a, device="cuda")[:, None])
        ref.close(got[at:at + a], *ref.attention(q[at:at + a], k, v, sees, scale or 1.0 / math.sqrt(hd), BF16_P, torch.bfloat16), (s, a, n, H, Hkv, hd))
        at += a
    assert bool((got[:first] == 5.0).all()) and bool((got[at:] == 5.0).all())


@pytest.mark.parametrize("hd", [16, 32, 64, 72, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 1), (6, 2), (14, 2), (32, 2), (80, 1)])
def test_cached_one_token(hd, H, Hkv):
    """One new token of each sequence, lengths around the page and none, more query heads per key head than a tile has rows."""
    bd = _bd()
    _cached_check(bd, [1] * 9, [1, 0, 63, 64, 65, 128, 300, 129, 7], H, Hkv, hd, True)


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_cached_several_tokens(hd, causal):
    """Several new tokens: tiles of rows that end inside a token's heads, more new tokens than held (the first see nothing), none."""
    bd = _bd()
    _cached_check(bd, [3, 0, 17, 5, 1], [200, 50, 17, 3, 0], 6, 2, hd, causal)
    _cached_check(bd, [64, 40, 130], [64, 100, 131], 3, 3, hd, causal, seed=3)
    _cached_check(bd, [300, 1], [333, 900], 8, 2, hd, causal, seed=4)


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_cached_long(hd, causal):
    """Long sequences, whose keys are split over blocks and joined; ragged, so that some splits are empty."""
    bd = _bd()
    _cached_check(bd, [1, 1, 1], [5000, 100, 3333], 8, 2, hd, causal)
    _cached_check(bd, [2, 20], [9001, 4000], 4, 4, hd, causal, seed=2, spread=3.0)
    _cached_check(bd, [70], [6400], 4, 1, hd, causal, seed=3, scale=0.3)


def test_cached_max_len():
    """A bound on the lengths: the same results where it holds, tokens beyond it left out where it does not."""
    bd = _bd()
    _cached_check(bd, [1, 1], [4000, 130], 4, 2, 64, True, max_len=4000)
    _cached_check(bd, [2, 3], [4000, 130], 4, 2, 64, False, max_len=1000)
    _cached_check(bd, [1, 1], [400, 30], 4, 2, 64, True, max_len=0)


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("new", [5, 40, 90])
def test_cached_hidden_values_have_no_part(hd, new):
    """A NaN in the value or key of one of the new tokens counts for it and the tokens behind it, not for those before it."""
    bd = _bd()
    H, Hkv, n = 4, 2, 150
    cache, table, _ = _fill(bd, [n], Hkv, hd)
    q = ref.randn((new, H, hd), torch.bfloat16, 9)
    run = lambda: bd.attention_cached(q, ref.starts_of([new]), cache, _dev(table), _dev([n]), causal=True)  # noqa: E731
    clean = run()
    at = n - new + new // 2
    page, place = int(table[0, at // 64]), at % 64
    for values in (True, False):
        pages = cache.v if values else cache.k
        old = pages.clone()
        if values:
            pages[page, :, 3, ref.PLACE[place]] = 0xFF
        else:
            pages[page, :, place, 3] = 0x7F
        got = run()
        pages.copy_(old)
        assert torch.equal(got[:new // 2], clean[:new // 2])
        rest = got[new // 2:]
        assert bool(rest[..., 3].isnan().all()) and (not values or torch.equal(rest[..., 4:], clean[new // 2:, :, 4:]))


def test_cached_scores_without_a_maximum():
    """Infinite queries: scores of -inf alone have no softmax; other rows are not touched by it."""
    bd = _bd()
    cache, table, _ = _fill(bd, [100], 1, 64)
    cache.k[int(table[0, 0]):int(table[0, 0]) + 1] = 0x38                  # 1.0 x scale everywhere
    cache.k[int(table[0, 1]):int(table[0, 1]) + 1] = 0x38
    q = ref.randn((2, 1, 64), torch.bfloat16, 1)
    clean = bd.attention_cached(q, ref.starts_of([2]), cache, _dev(table), _dev([100]), causal=False)
    q[1] = -math.inf
    got = bd.attention_cached(q, ref.starts_of([2]), cache, _dev(table), _dev([100]), causal=False)
    assert torch.equal(got[0], clean[0]) and bool(got[1].isnan().all())


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("H,tokens", [(4, 1), (4, 12), (8, 40)])
def test_cached_many_sequences(hd, H, tokens):
    """More sequences than a wave has lanes, long and short ones, with and without new tokens, in every height of tiles."""
    bd = _bd()
    rng = np.random.default_rng(tokens)
    lens = [int(n) for n in rng.integers(0, 200, 150)]
    lens[70], lens[149] = 6000, 2500
    new = [0 if s % 11 == 3 else int(rng.integers(1, 2 * tokens + 1)) if s % 5 else tokens for s in range(150)]
    _cached_check(bd, new, lens, H, 2, hd, True, seed=5)


@pytest.mark.parametrize("pad,offset", [(8, 8), (4, 4), (1, 0), (3, 5)])
@pytest.mark.parametrize("hd", [16, 32, 64, 72, 128])
def test_cached_many_rows_strides(pad, offset, hd):
    """Many rows per sequence with queries and outputs at any alignment and distance: the bits of contiguous ones."""
    bd = _bd()
    cache, table, _ = _fill(bd, [2000, 90], 2, hd)
    q = ref.randn((130, 8, hd), torch.bfloat16, 4)
    cu, held = ref.starts_of([50, 80]), _dev([2000, 90])
    plain = bd.attention_cached(q, cu, cache, _dev(table), held)
    strided = bd.attention_cached(ref.strided(q, pad, offset), cu, cache, _dev(table), held, out=ref.strided(torch.zeros_like(q), pad, offset))
    assert torch.equal(plain, strided)


@pytest.mark.parametrize("hd", [16, 32])
@pytest.mark.parametrize("causal", [False, True])
def test_cached_many_rows_of_small_heads(hd, causal):
    bd = _bd()
    _cached_check(bd, [70, 300, 1], [3000, 310, 64], 6, 2, hd, causal, seed=8)


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_cached_more_tiles_than_fit(hd, causal):
    """More tiles than the chip holds blocks, so that blocks end inside tiles: few long sequences, and many of which some are short, empty or
    without new tokens."""
    bd = _bd()
    _cached_check(bd, [2300, 30], [2400, 2000], 16, 16, hd, causal, seed=6)
    rng = np.random.default_rng(1)
    lens = [int(n) for n in rng.integers(0, 1500, 100)]
    lens[3], lens[99], lens[50] = 0, 1500, 40
    new = [0 if s % 13 == 5 else int(rng.integers(1, 80)) for s in range(100)]
    _cached_check(bd, new, lens, 24, 6, hd, causal, seed=7)


@pytest.mark.parametrize("hd", [64, 72, 128])
def test_cached_nan_where_blocks_end_inside_tiles(hd):
    """A NaN among the values reaches every row of its head that sees it, in whichever part of a tile it lies, and no other feature."""
    bd = _bd()
    H, n, new = 16, 2500, 2300
    cache, table, _ = _fill(bd, [n], H, hd)
    q = ref.randn((new, H, hd), torch.bfloat16, 9)
    run = lambda: bd.attention_cached(q, ref.starts_of([new]), cache, _dev(table), _dev([n]), causal=True)  # noqa: E731
    clean = run()
    for at in (3, 700, 1400, n - 1):
        page, place = int(table[0, at // 64]), ref.PLACE[at % 64]
        old = cache.v.clone()
        cache.v[page, 5, 7, place] = 0x7F
        got = run()
        cache.v.copy_(old)
        see = max(0, at - (n - new))                     # the first new token that sees it
        assert torch.equal(got[:see], clean[:see]) and torch.equal(got[:, :5], clean[:, :5]) and torch.equal(got[:, 6:], clean[:, 6:])
        assert bool(got[see:, 5, 7].isnan().all()) and torch.equal(got[:, 5, 8:], clean[:, 5, 8:]) and torch.equal(got[:, 5, :7], clean[:, 5, :7])


@pytest.mark.parametrize("hd", [64, 128])
def test_cached_one_and_many_tokens_in_one_call(hd):
    """Single tokens beside a whole prompt, and empty sequences alone."""
    bd = _bd()
    _cached_check(bd, [1, 700, 1, 0], [2000, 700, 65, 10], 4, 2, hd, True)
    _cached_check(bd, [0, 0], [100, 0], 4, 2, hd, True)


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("new", [2, 20, 200])
def test_cached_pages_that_are_none(hd, new):
    """Pages that are not held inside, at the start and at the end of a range, and more tokens than the table has room for, for every height
    of tiles; page 0, which belongs to nobody, holds NaN and so do its scales."""
    bd = _bd()
    Hkv, H, n = 1, 2, 40 * 64 + 90
    cache, table, _ = _fill(bd, [n, 64], Hkv, hd)
    table = table[:1].copy()
    table[0, [0, 5, 6, 7, 17, 39]] = [-1, 10 ** 6, cache.k.shape[0], -7, -2 ** 31, 2 ** 31 - 1]
    table = table[:, :40]
    free = [p for p in range(cache.k.shape[0]) if p not in table[0]]
    if 0 not in free:                                    # page 0 gives its place to a free one
        p = free[0]
        for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
            t[p] = t[0].clone()
        table[0, table[0] == 0] = p
    cache.k[0], cache.v[0] = 0x7F, 0xFF
    cache.k_scale[0], cache.v_scale[0] = math.nan, math.inf
    twin = ref.Cache(cache)
    q = ref.randn((new, H, hd), torch.bfloat16, 3)
    (k, held), (v, _) = twin.values(0, table[0], n), twin.values(1, table[0], n)
    assert not bool(held.all())
    for causal in (False, True):
        got = bd.attention_cached(q, ref.starts_of([new]), cache, _dev(table), _dev([n]), causal=causal)
        sees = held[None].expand(new, n)
        if causal:
            sees = sees & (torch.arange(n, device="cuda")[None] <= n - new + torch.arange(new, device="cuda")[:, None])
        ref.close(got, *ref.attention(q, k, v, sees, 1.0 / math.sqrt(hd), BF16_P, torch.bfloat16))


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("new", [5, 90])
def test_cached_nan_in_a_split_range(hd, new):
    """A NaN among the values of a long sequence reaches every row that sees it, whichever split holds it, and no other feature."""
    bd = _bd()
    H, Hkv, n = 4, 2, 5000
    cache, table, _ = _fill(bd, [n], Hkv, hd)
    q = ref.randn((new, H, hd), torch.bfloat16, 9)
    run = lambda: bd.attention_cached(q, ref.starts_of([new]), cache, _dev(table), _dev([n]), causal=True)  # noqa: E731
    clean = run()
    for at in (0, 2222, n - new, n - 1):
        page, place = int(table[0, at // 64]), ref.PLACE[at % 64]
        old = cache.v.clone()
        cache.v[page, 1, 7, place] = 0x7F
        got = run()
        cache.v.copy_(old)
        see = max(0, at - (n - new))                     # the first new token that sees it
        assert torch.equal(got[:see], clean[:see]) and torch.equal(got[:, :2], clean[:, :2])
        assert bool(got[see:, 2:, 7].isnan().all()) and torch.equal(got[..., 8:], clean[..., 8:]) and torch.equal(got[..., :7], clean[..., :7])


def test_cached_offsets_that_are_none():
    """Offsets that fall or leave the buffer reach nothing outside it."""
    bd = _bd()
    cache, table, _ = _fill(bd, [3000, 100, 64, 7, 900], 2, 64)
    pool = torch.full((120, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    q = ref.randn((100, 4, 64), torch.bfloat16, 1)
    for starts in ([0, 40, 10, 300, -5, 7], [90, 2 ** 31 - 1, -2 ** 31, 100, 0, 100]):
        bd.attention_cached(q, _dev(starts), cache, _dev(table), _dev([3000, 100, 64, 7, 900]), out=pool[10:110])
        assert bool((pool[:10] == 5.0).all()) and bool((pool[110:] == 5.0).all())


def test_cache_beyond_32_bits():
    """Pages whose bytes lie more than 2^32 behind the first, in every call."""
    bd = _bd()
    heads, hd, pages = 8, 128, 66000                    # 4.3 GB of keys and as much of values
    cache = bd.KVCache.empty(pages, heads, hd)
    near = bd.KVCache.empty(8, heads, hd)
    far, close = [pages - 1, 65999 - 7, 65537], [0, 3, 5]
    n = 150
    k, v = ref.randn((n, heads, hd), torch.bfloat16, 1), ref.randn((n, heads, hd), torch.bfloat16, 2)
    got = []
    for c, t in ((cache, far), (near, close)):
        table = _dev([t])
        bd.kv_store(c, table, _dev([0]), k, v, ref.starts_of([n]))
        out = [*bd.kv_load(c, table, _dev([0]), ref.starts_of([n]), n, torch.bfloat16)]
        for new in (1, 40, 140):
            q = ref.randn((new, 8, hd), torch.bfloat16, 3)
            out.append(bd.attention_cached(q, ref.starts_of([new]), c, table, _dev([n])))
        got.append(out)
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert float((got[0][0] - k).abs().max()) <= 2.0 ** -4 * float(k.abs().max())


# ---- together -----------------------------------------------------------------------------------------------


def test_together_frame_by_frame():
    """Two clips, frame by frame, as a program runs them: turn q and k, store k and v, attend over everything stored.  Against 64-bit
    attention over the values the cache holds; and the last frames against packed attention over those values."""
    bd = _bd()
    H, Hkv, hd, dims = 8, 4, 128, (16, 56, 56)
    grids, frames = [(6, 7), (4, 5)], 4
    sizes = [h * w for h, w in grids]
    cache = _new_cache(bd, 12, Hkv, hd)
    table = _tables(12, [3, 2], 3)
    past = np.zeros(2, np.int64)
    rope = bd.make_rope(dims)
    for f in range(frames):
        pos = torch.tensor([[f, i, j] for h, w in grids for i in range(h) for j in range(w)], dtype=torch.int32, device="cuda")
        qkv = ref.randn((sum(sizes), (H + 2 * Hkv) * hd), torch.bfloat16, 100 + f)
        q, k, v = qkv[:, :H * hd].view(-1, H, hd), qkv[:, H * hd:(H + Hkv) * hd].view(-1, Hkv, hd), qkv[:, (H + Hkv) * hd:].view(-1, Hkv, hd)
        norm = 1.0 + ref.randn((hd,), torch.bfloat16, 7, 0.1)
        bd.rope_axes(rope, pos, q, k, norm, norm, out=(q, k))
        starts = ref.starts_of(sizes)
        bd.kv_store(cache, _dev(table), _dev(past), k, v, starts)
        past += sizes
        out = bd.attention_cached(q, starts, cache, _dev(table), _dev(past), causal=False)
        twin = ref.Cache(cache)
        at = 0
        for s, n in enumerate(sizes):
            (kk, held), (vv, _) = twin.values(0, table[s], int(past[s])), twin.values(1, table[s], int(past[s]))
            ref.close(out[at:at + n], *ref.attention(q[at:at + n], kk, vv, held[None].expand(n, -1), 1 / math.sqrt(hd), BF16_P, torch.bfloat16), (f, s))
            at += n
    everything = ref.starts_of(past.tolist())
    kk, vv = bd.kv_load(cache, _dev(table), _dev([0, 0]), everything, int(past.sum()), torch.bfloat16)
    whole = torch.zeros((int(past.sum()), H, hd), dtype=torch.bfloat16, device="cuda")
    ends = np.cumsum(past)
    for s, n in enumerate(sizes):
        whole[ends[s] - n:ends[s]] = q[sum(sizes[:s]):sum(sizes[:s]) + n]
    packed = bd.attention_packed(whole, kk, vv, everything)
    for s, n in enumerate(sizes):
        a, b = packed[ends[s] - n:ends[s]].double(), out[sum(sizes[:s]):sum(sizes[:s]) + n].double()
        # each is within one rounding of P and one of the result, of sum p |v| <= max |v|
        assert float((a - b).abs().max()) <= 4 * 2.0 ** -8 * float(vv.abs().max())


def _chain(bd):
    """The calls of one step on static tensors, for streams and graphs: returns (inputs, cache, run)."""
    H, Hkv, hd = 8, 2, 64
    lens, past = [5, 130, 1], [100, 0, 4000]
    cache = bd.KVCache.empty(80, Hkv, hd)
    table = _dev(_tables(80, [2, 3, 63], 63))
    x = ref.randn((136, (H + 2 * Hkv) * hd), torch.bfloat16, 1)
    q, k, v = x[:, :H * hd].view(-1, H, hd), x[:, H * hd:(H + Hkv) * hd].view(-1, Hkv, hd), x[:, (H + Hkv) * hd:].view(-1, Hkv, hd)
    pos = torch.arange(136 * 2, device="cuda", dtype=torch.int32).view(136, 2)
    starts, at, held = ref.starts_of(lens), _dev(past), _dev([105, 130, 4001])
    rope = bd.make_rope((32, 32))

    def run():
        qr, kr = bd.rope_axes(rope, pos, q, k)
        bd.kv_store(cache, table, at, kr, v, starts)
        return (bd.attention_packed(qr, kr, v, starts, causal=True), bd.attention_cached(qr, starts, cache, table, held),
                *bd.kv_load(cache, table, at, starts, 136, torch.bfloat16))
    return x, run


def test_on_another_stream():
    bd = _bd()
    x, run = _chain(bd)
    want = run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run()
    s.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_two_streams_at_once():
    """Two chains with caches of their own, in turn on two streams without a wait between."""
    bd = _bd()
    chains = [_chain(bd) for _ in range(2)]
    chains[1][0].copy_(ref.randn(tuple(chains[1][0].shape), torch.bfloat16, 77))
    want = [run() for _, run in chains]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in chains]
    for turn in range(8):
        got = []
        for (_, run), s in zip(chains, streams):
            with torch.cuda.stream(s):
                got.append(run())
        for s in streams:
            s.synchronize()
        for a, b in zip(want, got):
            for x, y in zip(a, b):
                assert torch.equal(x, y), turn


def test_captured_and_replayed():
    """A graph of the whole chain (two of them, alive together, with workspaces of their own), replayed with new inputs and eager work between."""
    bd = _bd()
    x, run = _chain(bd)
    run()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out))
    for turn in range(4):
        x.copy_(ref.randn(tuple(x.shape), torch.bfloat16, 10 + turn))
        want = run()
        torch.cuda.synchronize()
        for g, out in graphs:
            for o in out:
                o.zero_()
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(want, out):
                assert torch.equal(a, b), turn


def test_captured_step_replayed_over_growing_sequences():
    """One graph of a step of single tokens, replayed while the lists on the device grow past page ends: each time the bits of an eager step."""
    bd = _bd()
    H, Hkv, hd, n = 8, 2, 128, 3
    table = _dev(_tables(60, [20, 20, 20], 20))
    lens = [62, 0, 1150]
    caches = [bd.KVCache.empty(60, Hkv, hd) for _ in range(2)]
    k, v = ref.randn((sum(lens), Hkv, hd), torch.bfloat16, 1), ref.randn((sum(lens), Hkv, hd), torch.bfloat16, 2)
    for c in caches:
        bd.kv_store(c, table, _dev([0] * n), k, v, ref.starts_of(lens))
    x = ref.randn((n, H + 2 * Hkv, hd), torch.bfloat16, 3)
    starts, past, held = ref.starts_of([1] * n), _dev(lens), _dev(lens) + 1
    pos = past[:, None].clone()
    rope = bd.make_rope((hd,), pairing=bd.ROPE_HALVES)

    def step(cache):
        q, kk = bd.rope_axes(rope, pos, x[:, :H], x[:, H:H + Hkv])
        bd.kv_store(cache, table, past, kk, x[:, H + Hkv:], starts)
        return bd.attention_cached(q, starts, cache, table, held)
    scratch = bd.KVCache.empty(60, Hkv, hd)
    step(scratch)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(caches[0])
    for turn in range(6):
        x.copy_(ref.randn(tuple(x.shape), torch.bfloat16, 10 + turn))
        want = step(caches[1])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and not bool(out.isnan().any()), turn
        for a, b in zip((caches[0].k, caches[0].v, caches[0].k_scale, caches[0].v_scale), (caches[1].k, caches[1].v, caches[1].k_scale, caches[1].v_scale)):
            assert torch.equal(a, b), turn
        for t in (past, held, pos):
            t += 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_rope_features_that_stay(dtype, halves, normed):
    """Features behind those that turn are neither turned nor mixed: infinities, NaN and -0 among them stay where they are."""
    bd = _bd()
    dt, tokens, H = _dt(dtype), 9, 5
    # four pairs a lane, rotations that end inside a lane, one pair a lane (heads of 30, views off their alignment)
    for hd, dims, pad, offset in ((72, (32, 32), 0, 0), (128, (64,), 0, 0), (64, (10, 6), 0, 0), (72, (12, 2), 0, 0), (30, (6, 10), 0, 0), (72, (32, 32), 1, 1)):
        R, g = sum(dims), torch.Generator(device="cuda").manual_seed(hd)
        x = ref.randn((tokens, H, hd), dt, hd + R)
        for i, bad in enumerate((math.inf, -math.inf, math.nan, -0.0, -0.0)):
            x[i, i % H, R + 2 * i % (hd - R)] = bad                 # even and odd ones: either side of what would be a pair
            x[i + 2, (i + 1) % H, R + (2 * i + 1) % (hd - R)] = bad
        x[8, :, R:] = -0.0
        pos = torch.randint(0, 1000, (tokens, len(dims)), generator=g, device="cuda", dtype=torch.int32)
        norm = 1.0 + ref.randn((hd,), dt, 3, 0.1) if normed else None
        rope = bd.make_rope(dims, pairing=bd.ROPE_HALVES if halves else bd.ROPE_ADJACENT)
        if pad or offset:
            x = ref.strided(x, pad, offset)
        for got in (bd.rope_axes(rope, pos, x, q_norm=norm), bd.rope_axes(rope, pos, x.clone(), x, norm, norm)[1]):
            want, tol = ref.rope(x, pos, dims, [10000.0] * 2, [1.0] * 2, halves, False, norm, 1e-6)
            number = want.isfinite()
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf()), (hd, dims)
            assert bool((((got.double() - want).abs() <= tol) | ~number).all()), (hd, dims)
            assert torch.equal(got[..., R:].signbit() & number[..., R:], want[..., R:].signbit() & number[..., R:]), (hd, dims)
            if not normed:
                assert bool(((got[..., R:] == x[..., R:]) | x[..., R:].isnan()).all()), (hd, dims)


@pytest.mark.parametrize("n", [250, 255, 256])
def test_cached_one_long_among_many_short(n):
    """About as many single tokens as four rounds of blocks take, one of them over a long sequence."""
    bd = _bd()
    lens = [500 - s % 3 for s in range(n)]
    lens[n // 2] = 512 * 64 - 5
    _cached_check(bd, [1] * n, lens, 8, 8, 64, True, seed=4)


@pytest.mark.parametrize("hd", [64, 72, 128])
@pytest.mark.parametrize("new,lens,max_len", [([3, 5], [200, 150], 148), ([14, 9], [300, 150], 146), ([70, 90], [300, 260], 200), ([40], [4000], 3990), ([4, 1], [4000, 2000], 1997)])
def test_cached_causal_bound_below_the_lengths(hd, new, lens, max_len):
    """max_len cuts sequences off inside the new tokens, and well before them; what a new token sees follows from its place in the whole
    sequence all the same.  Tiles of 16, 32 and 128 rows, split and not."""
    bd = _bd()
    H, Hkv = 4, 2
    cache, table, twin = _fill(bd, lens, Hkv, hd, 11)
    q = ref.randn((sum(new), H, hd), torch.bfloat16, 12)
    got, at = bd.attention_cached(q, ref.starts_of(new), cache, _dev(table), _dev(lens), causal=True, max_len=max_len), 0
    for s, (a, n) in enumerate(zip(new, lens)):
        (k, held), (v, _) = twin.values(0, table[s], n), twin.values(1, table[s], n)
        key = torch.arange(n, device="cuda")[None]
        sees = held[None] & (key < max_len) & (key <= n - a + torch.arange(a, device="cuda")[:, None])
        ref.close(got[at:at + a], *ref.attention(q[at:at + a], k, v, sees, 1.0 / math.sqrt(hd), BF16_P, torch.bfloat16), (s, a, n))
        at += a


@pytest.mark.parametrize("total", [3, 45, 200])
def test_captured_attention_over_lists_that_change(total):
    """One graph of attention over a table wide enough to be split, for every height of tiles: between its replays the lists on the device
    change how the work is dealt (nothing split, one sequence split, all of them), and so do the tokens' sequences.  Each time the bits of an eager call."""
    bd = _bd()
    H, Hkv, hd, width, n = 8, 2, 128, 160, 3
    table = _dev(_tables(3 * width, [width] * n, width))
    cache = bd.KVCache.empty(3 * width, Hkv, hd)
    rows = width * 64
    for s in range(n):
        k, v = ref.randn((rows, Hkv, hd), torch.bfloat16, 2 * s), ref.randn((rows, Hkv, hd), torch.bfloat16, 2 * s + 1)
        bd.kv_store(cache, table[s:s + 1], _dev([0]), k, v, ref.starts_of([rows]))
    q = ref.randn((total, H, hd), torch.bfloat16, 9)
    third = total // 3
    turns = [([0, third, 2 * third, total], [62, 0, 1150]), ([0, third, 2 * third, total], [70, 9001, 1151]), ([0, third, 2 * third, total], [rows, rows - 1, rows - 63]),
             ([0, 0, 1, total], [rows, 5000, 300]), ([0, total, total, total], [rows, 17, 0]), ([0, third, 2 * third, total], [63, 1, 1151])]
    starts, held = _dev(turns[0][0]), _dev(turns[0][1])
    bd.attention_cached(q, starts, cache, table, held)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = bd.attention_cached(q, starts, cache, table, held)
    for turn, (a, b) in enumerate(turns):
        starts.copy_(_dev(a))
        held.copy_(_dev(b))
        want = bd.attention_cached(q, starts, cache, table, held)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and not bool(out.isnan().any()), turn
        for s in range(n):
            if a[s + 1] > a[s] and b[s] == 0:
                assert bool((out[a[s]:a[s + 1]] == 0).all())


@pytest.mark.parametrize("max_len", [2 ** 31, 2 ** 32, 2 ** 32 + 70, 2 ** 40])
def test_cached_bound_beyond_32_bits(max_len):
    """A bound that no sequence reaches, however large: the bits without one."""
    bd = _bd()
    cache, table, _ = _fill(bd, [1500, 90], 2, 64)
    q = ref.randn((4, 4, 64), torch.bfloat16, 1)
    call = [q, ref.starts_of([3, 1]), cache, _dev(table), _dev([1500, 90])]
    assert torch.equal(bd.attention_cached(*call, max_len=max_len), bd.attention_cached(*call))
    with pytest.raises(bd.SpecaError):
        bd.attention_cached(*call, max_len=-max_len)


@pytest.mark.parametrize("hd", [64, 72])
@pytest.mark.parametrize("H,Hkv", [(8, 8), (16, 16), (24, 24), (16, 8), (48, 16)])
def test_packed_key_heads_by_the_eight(hd, H, Hkv):
    """As many key heads as there are XCDs, and multiples: every head gets its own keys however heads are dealt."""
    bd = _bd()
    for causal in (False, True):
        _packed_check(bd, [130, 3, 77], H, Hkv, hd, "bf16", causal, seed=3)
