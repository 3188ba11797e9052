"""Refusals of the operators around attention, all of them decided on the host ahead of any GPU work, and their workspace sizes."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def bd():
    from paper_2509_11628_amd import binding
    binding.load_library()
    return binding


A = 1 << 20          # an address that is never followed: every call below is refused, or has no tokens


def _code(bd, name, *args):
    lib = bd.load_library()
    code = getattr(lib, name)(None, *args)
    if code != bd.OK:
        assert lib.speca_last_error(None).decode().startswith(name), lib.speca_last_error(None)
    return code


def _rope(bd, dtype=1, tokens=3, hd=64, eps=1e-6, positions=A, q=(A, A, None, 256, 256, 4), k=None, **fields):
    r = bd.make_rope((32, 32))
    for n, v in fields.items():
        if n in ("dims", "theta", "scale"):
            for i, x in enumerate(v):
                getattr(r, n)[i] = x
        else:
            setattr(r, n, v)
    return _code(bd, "speca_rope_axes", dtype, r, positions, tokens, hd, eps, bd.RopeIO(*q), bd.RopeIO(*k) if k else None)


def test_rope_refusals(bd):
    assert _rope(bd, tokens=0) == bd.OK
    for bad in (dict(dtype=7), dict(tokens=-1), dict(tokens=1 << 31), dict(hd=63), dict(hd=0), dict(hd=130), dict(hd=32), dict(eps=-1.0), dict(eps=float("nan")), dict(positions=None),
                dict(axes=0), dict(axes=5), dict(dims=(31,)), dict(dims=(0,)), dict(dims=(-2,)), dict(dims=(66,)), dict(theta=(0.0,)), dict(theta=(float("inf"),)),
                dict(scale=(float("nan"),)), dict(pairing=2), dict(spectrum=-1), dict(q=(None, A, None, 256, 256, 4)), dict(q=(A, None, None, 256, 256, 4)),
                dict(q=(A, A, None, 255, 256, 4)), dict(q=(A, A + 64, None, 256, 200, 4)), dict(q=(A, A, None, 256, 512, 4)), dict(q=(A + 1, A, None, 256, 256, 4)),
                dict(q=(A, A, A + 1, 256, 256, 4)), dict(q=(A, A, None, 256, 256, 0)), dict(k=(None, A, None, 256, 256, 4)), dict(k=(A, A, None, 256, 256, 70000))):
        assert _rope(bd, **bad) == bd.EINVAL, bad
    lib = bd.load_library()
    assert lib.speca_rope_axes(None, 1, None, A, 3, 64, 1e-6, bd.RopeIO(A, A, None, 256, 256, 4), None) == bd.EINVAL
    assert lib.speca_rope_axes(None, 1, bd.make_rope((32,)), A, 3, 64, 1e-6, None, None) == bd.EINVAL
    with pytest.raises(ValueError):
        bd.make_rope(())
    with pytest.raises(ValueError):
        bd.make_rope((8, 8), theta=(1.0,))


def _packed(bd, dtype=1, q=A, ldq=256, k=A, ldk=128, v=A, ldv=128, out=A, ldo=256, starts=A, n=2, total=10, heads=4, kv=2, hd=64, causal=0, scale=0.0):
    return _code(bd, "speca_attention_packed", dtype, q, ldq, k, ldk, v, ldv, out, ldo, starts, n, total, heads, kv, hd, causal, scale)


def test_packed_refusals(bd):
    assert _packed(bd, total=0) == bd.OK
    for bad in (dict(dtype=2), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(starts=None), dict(n=0), dict(total=-1), dict(heads=0), dict(kv=0), dict(kv=3),
                dict(heads=70000, kv=1, ldq=1 << 23, ldo=1 << 23), dict(ldq=255), dict(ldo=255), dict(ldk=127), dict(ldv=127), dict(ldk=1 << 50), dict(q=A + 1), dict(out=A + 1),
                dict(starts=A + 2), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(total=0x7FFFFFFF, heads=65536, kv=65536, ldq=1 << 22, ldk=1 << 22, ldv=1 << 22, ldo=1 << 22)):
        assert _packed(bd, **bad) == bd.EINVAL, bad
    for hd in (8, 48, 96, 256):
        assert _packed(bd, hd=hd, ldq=2048, ldk=2048, ldv=2048, ldo=2048) == bd.EUNSUPPORTED


def _cache(bd, k=A, v=A, ks=A, vs=A, pages=8, heads=2, hd=64):
    return bd.KVCacheDesc(k, v, ks, vs, pages, heads, hd)


@pytest.mark.parametrize("name", ["speca_kv_store", "speca_kv_load"])
def test_store_and_load_refusals(bd, name):
    def call(dtype=1, cache=None, table=(A, 4), first=A, k=A, ldk=128, v=A, ldv=128, starts=A, n=2, total=10):
        return _code(bd, name, dtype, _cache(bd, **(cache or {})), bd.KVTable(*table), first, k, ldk, v, ldv, starts, n, total)

    assert call(total=0) == bd.OK
    for bad in (dict(dtype=5), dict(first=None), dict(k=None), dict(v=None), dict(starts=None), dict(n=0), dict(total=-4), dict(ldk=127), dict(ldv=100), dict(ldv=1 << 60),
                dict(k=A + 1), dict(first=A + 1), dict(starts=A + 3), dict(table=(None, 4)), dict(table=(A, 0)), dict(table=(A + 1, 4)),
                dict(cache=dict(k=None)), dict(cache=dict(v=None)), dict(cache=dict(ks=None)), dict(cache=dict(vs=None)), dict(cache=dict(k=A + 8)), dict(cache=dict(v=A + 4)),
                dict(cache=dict(ks=A + 1)), dict(cache=dict(pages=0)), dict(cache=dict(heads=0)), dict(total=0x7FFFFFFF, cache=dict(heads=60000), ldk=1 << 22, ldv=1 << 22)):
        assert call(**bad) == bd.EINVAL, bad
    assert call(cache=dict(hd=80), ldk=1024, ldv=1024) == bd.EUNSUPPORTED
    lib = bd.load_library()
    assert getattr(lib, name)(None, 1, None, bd.KVTable(A, 4), A, A, 128, A, 128, A, 2, 10) == bd.EINVAL
    assert getattr(lib, name)(None, 1, _cache(bd), None, A, A, 128, A, 128, A, 2, 10) == bd.EINVAL


def test_cached_refusals(bd):
    def call(dtype=1, q=A, ldq=256, out=A, ldo=256, starts=A, n=2, total=10, cache=None, table=(A, 400), lens=A, max_len=100, heads=4, causal=1, scale=0.0, room=None, size=0):
        return _code(bd, "speca_attention_cached", dtype, q, ldq, out, ldo, starts, n, total, _cache(bd, **(cache or {})), bd.KVTable(*table), lens, max_len, heads, causal, scale, room, size)

    assert call(total=0) == bd.OK
    assert call(dtype=0) == bd.EUNSUPPORTED
    assert call(cache=dict(hd=96), ldq=1024, ldo=1024) == bd.EUNSUPPORTED
    for bad in (dict(dtype=9), dict(q=None), dict(out=None), dict(starts=None), dict(lens=None), dict(n=0), dict(total=-1), dict(max_len=-1), dict(max_len=(1 << 30) + 1), dict(heads=0),
                dict(heads=3), dict(ldq=255), dict(ldo=10), dict(q=A + 1), dict(out=A + 1), dict(lens=A + 2), dict(scale=-0.5), dict(scale=float("inf")), dict(cache=dict(k=A + 2)),
                dict(table=(A, 0)), dict(total=0x7FFFFFFF, heads=65536, cache=dict(heads=1), ldq=1 << 23, ldo=1 << 23)):
        assert call(**bad) == bd.EINVAL, bad
    size = bd.load_library().speca_attention_cached_workspace(2, 10, 20000, 4, 2, 64)
    assert size > 0 and size % 16 == 0
    for room, given in ((None, size), (A, size - 1), (A + 8, size)):
        assert call(max_len=20000, room=room, size=given) == bd.EINVAL


def test_cached_workspace_sizes(bd):
    f = bd.load_library().speca_attention_cached_workspace
    assert f(4, 4, 64, 32, 8, 128) == 0 and f(4, 0, 100000, 32, 8, 128) == 0
    for bad in ((0, 1, 1, 1, 1, 64), (1, -1, 1, 1, 1, 64), (1, 1, -1, 1, 1, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 0, 1, 64), (1, 1, 1, 1, 1, 40)):
        assert f(*bad) == -1
    rng = np.random.default_rng(0)
    for _ in range(300):
        n, total, longest = int(rng.integers(1, 300)), int(rng.integers(1, 5000)), int(rng.integers(0, 200000))
        kv = int(rng.integers(1, 25)); heads = kv * int(rng.integers(1, 17))
        size = f(n, total, longest, heads, kv, 128)
        # sums and statistics of every split of every row tile: bounded by a few times what the queries of a full chip need
        assert 0 <= size < 1 << 32 and size % 16 == 0


def test_binding_refuses_what_does_not_fit(bd):
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        bd.attention_packed(q, q, q, torch.zeros(2, dtype=torch.int32))          # not on a device
    with pytest.raises(ValueError):
        bd.rope_axes(bd.make_rope((32,)), torch.zeros((4, 1), dtype=torch.int32), q)
    with pytest.raises(ValueError):
        bd.KVCache(torch.zeros((2, 1, 32, 64), dtype=torch.uint8), torch.zeros((2, 1, 64, 64), dtype=torch.uint8), torch.ones((2, 1)), torch.ones((2, 1)))


def test_operator_struct_layouts(bd):
    assert C.sizeof(bd.Rope) == 4 * 15 and C.sizeof(bd.RopeIO) == 48 and C.sizeof(bd.KVCacheDesc) == 48 and C.sizeof(bd.KVTable) == 16


def test_misaligned_lists_are_refused(bd):
    assert _rope(bd, positions=A + 2) == bd.EINVAL
    assert _packed(bd, starts=A + 2) == bd.EINVAL


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_how_few_rows_are_cut(tmp_path):
    """csrc/deal.h on the host: no cliff in the number of sequences, no more units than the workspace has room for, sums beyond 32 bits."""
    exe = str(tmp_path / "deal")
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", os.path.join(here, "deal_driver.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "dealing is right" in r.stdout, r.stdout + r.stderr


def test_more_blocks_than_a_launch_has_are_refused(bd):
    """2^32 threads and more along one dimension are no launch: refused ahead of it, as the argument that it is."""
    wide = 128 * 64
    assert _rope(bd, tokens=1 << 26) == bd.EINVAL
    for dtype in (0, 1):
        assert _packed(bd, dtype=dtype, total=1 << 24, heads=128, kv=128, ldq=wide, ldk=wide, ldv=wide, ldo=wide) == bd.EINVAL
    for name in ("speca_kv_store", "speca_kv_load"):
        assert _code(bd, name, 1, _cache(bd, heads=128), bd.KVTable(A, 4), A, A, wide, A, wide, A, 2, 1 << 23) == bd.EINVAL
    for n, total in ((2, 1 << 26), (1 << 21, 1 << 21), (1 << 20, 1 << 24)):
        room = bd.load_library().speca_attention_cached_workspace(n, total, 20000, 64, 64, 64)
        assert _code(bd, "speca_attention_cached", 1, A, 4096, A, 4096, A, n, total, _cache(bd, heads=64), bd.KVTable(A, 400), A, 20000, 64, 1, 0.0, A, room) == bd.EINVAL
        assert "too many" in bd.load_library().speca_last_error(None).decode()


def test_sizes_beyond_32_bits_are_refused_by_the_binding(bd):
    """The library takes sizes as int: what does not fit is refused, not cut off."""
    like = torch.empty((4, 2, 64), dtype=torch.bfloat16, device="meta")
    for shape in ((2 ** 32 + 5, 2, 64), (2 ** 31, 2, 64), (4, 2 ** 32 + 2, 64)):
        with pytest.raises(ValueError):
            bd._heads("q", torch.empty(shape, dtype=torch.bfloat16, device="meta"), like)
    for shape in ((2 ** 32 + 3,), (2 ** 31,)):
        with pytest.raises(ValueError):
            bd._ints("starts", torch.empty(shape, dtype=torch.int32, device="meta"), like, 1)
    with pytest.raises(ValueError):
        bd._ints("table", torch.empty((2, 2 ** 32 + 1), dtype=torch.int32, device="meta"), like, 2, 2)
    assert bd._heads("q", torch.empty((2 ** 31 - 1, 2, 64), dtype=torch.bfloat16, device="meta"), like) == 128
