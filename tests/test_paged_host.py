"""The serving operators without a GPU: what is refused before any HIP call, the rules of the launch, the product that stands for a division."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import paper_2501_08071_amd as P

HERE = os.path.dirname(os.path.abspath(__file__))
OK = 4096      # any 16-byte aligned address: validation fails before it is touched


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    out = str(tmp_path_factory.mktemp("paged_launch") / "paged_launch_host.so")
    res = subprocess.run([gxx, "-std=c++20", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-isystem", "/opt/rocm/include",
                          os.path.join(HERE, "csrc", "paged_launch_host.cpp"), "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return ctypes.CDLL(out)


def plan(L, *args):
    out = (ctypes.c_longlong * 11)()
    L.plan(*args, out)
    return dict(zip("rows workgroups balanced direct waves prefix_rows prefix_tiles prefix_splits bytes part_floats prefix_floats".split(), out))


def test_division_by_a_product(L):
    top = 2 ** 31 - 1
    for d in list(range(1, 300)) + [1 << k for k in range(9, 29)] + [(1 << k) + 1 for k in range(9, 28)] + [(1 << k) - 1 for k in range(9, 29)]:
        for q in {0, 1, 2, 77, top // d - 1, top // d}:
            for n in (q * d - 1, q * d, q * d + 1, q * d + d - 1):
                if 0 <= n <= top:
                    assert L.divided(n, d) == n // d, (n, d)


def test_launches_hold_every_tile_and_their_work_fits(L):
    r = random.Random(3)
    for _ in range(3000):
        Hk = r.choice([1, 2, 3, 8, 64])
        G, D, B = r.choice([1, 2, 4, 5, 16, 20, 64]), r.choice([32, 64, 128]), r.choice([1, 2, 7, 64, 300, 5000])
        new = [r.choice([0, 1, 1, 1, 3, 8, r.randrange(1, 3000)]) for _ in range(min(B, 40))] + [1] * (B - min(B, 40))
        T, max_q, max_kv, pre = sum(new), max(new), r.choice([0, 1, 300, 5000, 1 << 17, 1 << 30]), r.choice([0, 0, 1, 100, 5000, 1 << 20])
        if T == 0:
            continue
        p = plan(L, B, T, Hk * G, Hk, D, max_q, max_kv, pre)
        tiles = sum(-(-n * G // p["rows"]) for n in new) * Hk
        if p["direct"]:
            assert max_q * G <= p["rows"] and p["workgroups"] == B * Hk
        elif not p["balanced"]:
            assert p["workgroups"] >= tiles
        else:
            assert p["workgroups"] in (256, 512) and tiles * (max_kv // (32 if p["rows"] < 128 and D == 128 else 64) + 13) < 2 ** 31
            assert p["part_floats"] >= 2 * p["workgroups"] * p["rows"] * (D + 2) + 8 * p["workgroups"]
        assert 1 <= p["workgroups"] <= 1 << 24 and p["workgroups"] * 64 * p["waves"] < 2 ** 32
        assert (p["prefix_splits"] > 0) == (pre > 0)
        if pre:
            assert p["prefix_tiles"] * p["prefix_rows"] >= T * G and p["prefix_splits"] <= max(1, pre // 32)
            assert p["prefix_floats"] >= p["prefix_splits"] * T * Hk * G * (D + 2) and p["prefix_floats"] % 4 == 0
            assert p["prefix_tiles"] * Hk * p["prefix_splits"] * 512 < 2 ** 32
        assert p["bytes"] == 4 * (p["part_floats"] + p["prefix_floats"]) == P.attn_paged_workspace(B, T, Hk * G, Hk, D, max_q, max_kv, pre)


def cache(**x):
    c = P.PagedCache(OK, OK, 8 * 16 * 64, 10, 16, 8, 64, 0, OK, 4, 4, OK, OK, 2, 3)
    for n, v in x.items():
        setattr(c, n, v)
    return c


BAD_CACHES = [(-3, dict(dtype=2)), (-3, dict(dtype=-1)), (-2, dict(B=-1)), (-2, dict(T=-1)), (-2, dict(T=1 << 23)), (-2, dict(B=1 << 21)), (-2, dict(Hk=0)),
              (-5, dict(D=96)), (-2, dict(D=0)), (-2, dict(page_size=0)), (-2, dict(page_size=24)), (-2, dict(page_size=-16)), (-2, dict(n_pages=-1)),
              (-2, dict(n_pages=0)), (-2, dict(width=-1)), (-2, dict(table_stride=3)), (-2, dict(width=1 << 28, table_stride=1 << 28)),
              (-2, dict(page_stride=8 * 16 * 64 - 8)), (-2, dict(page_stride=8 * 16 * 64 + 4)), (-2, dict(page_stride=1 << 40)), (-1, dict(k=None)),
              (-1, dict(v=None)), (-1, dict(page_table=None)), (-1, dict(cu_q=None)), (-1, dict(kv_len=None)), (-7, dict(k=OK + 8)), (-7, dict(v=OK + 2)),
              (-7, dict(page_table=OK + 2)), (-7, dict(cu_q=OK + 1)), (-7, dict(kv_len=OK + 2))]


def fwd(c=None, q=OK, qs=16 * 64, o=OK, lse=OK, pt=0, pl=0, Hq=16, mq=2, mk=100, scale=1.0, ws=OK, n=1 << 30):
    return P.attn_paged_fwd_raw(c or cache(), q, qs, o, lse, pt, pl, Hq, mq, mk, scale, ws, n, 0)


def append(c=None, q=OK, k=OK, v=OK, qs=16 * 64, ks=8 * 64, vs=8 * 64, out=OK, cos=OK, sin=OK, rot=64, il=0, n=100, off=0, Hq=16):
    return P.attn_kv_append_raw(c or cache(), q, k, v, qs, ks, vs, out, cos, sin, rot, il, n, off, Hq, 0)


def test_bad_arguments_are_refused():
    for status, x in BAD_CACHES:
        assert fwd(cache(**x)) == status, x
        assert append(cache(**x)) == status, x
    assert P.lib.attn_paged_fwd(None, OK, 0, OK, OK, None, 0, 16, 1, 1, 1.0, None, 0, None) == -1
    assert P.lib.attn_kv_append(None, OK, OK, OK, 0, 0, 0, OK, None, None, 0, 0, 0, 0, 16, None) == -1
    assert fwd(q=0) == -1 and fwd(o=0) == -1 and fwd(pl=5) == -1
    assert fwd(Hq=0) == -2 and fwd(Hq=12) == -2 and fwd(mq=-1) == -2 and fwd(mk=-1) == -2 and fwd(pl=-1) == -2 and fwd(qs=-8) == -2 and fwd(qs=12) == -2
    assert fwd(scale=float("nan")) == -4 and fwd(scale=float("inf")) == -4
    assert fwd(q=OK + 2) == -7 and fwd(o=OK + 8) == -7 and fwd(lse=OK + 2) == -7 and fwd(ws=OK + 8) == -7
    need = P.attn_paged_workspace(2, 3, 16, 8, 64, 2, 100000, 77)
    assert need > 0 and fwd(mk=100000, pt=OK, pl=77, n=need - 1) == -8 and fwd(mk=100000, pt=OK, pl=77, ws=0) == -8
    assert P.attn_paged_workspace(2, 3, 16, 8, 64, 2, 100, 0) == 0
    for bad in ((-1, 3, 16, 8, 64, 2, 9, 0), (2, -3, 16, 8, 64, 2, 9, 0), (2, 3, 15, 8, 64, 2, 9, 0), (2, 3, 16, 8, 96, 2, 9, 0), (2, 3, 16, 8, 64, -2, 9, 0),
                (2, 3, 16, 8, 64, 2, -9, 0), (2, 3, 16, 8, 64, 2, 9, -1), (2, 3, 0, 8, 64, 2, 9, 0), (2, 1 << 22, 256, 8, 64, 2, 9, 0)):
        assert P.attn_paged_workspace(*bad) == -1
    assert append(k=0) == -1 and append(v=0) == -1 and append(q=0) == -1 and append(out=0) == -1 and append(cos=0) == -1 and append(sin=0) == -1
    assert append(rot=-16) == -2 and append(rot=80) == -2 and append(rot=24) == -2 and append(n=0) == -2 and append(ks=4) == -2 and append(vs=-8) == -2 and append(Hq=-1) == -2
    assert append(q=OK + 4) == -7 and append(k=OK + 8) == -7 and append(v=OK + 8) == -7 and append(out=OK + 8) == -7 and append(cos=OK + 4) == -7
    # nothing to do: valid, and nothing is launched
    for x in (dict(T=0), dict(B=0)):
        assert fwd(cache(**x, k=None, cu_q=None), q=0, o=0, ws=0) == 0 and append(cache(**x, k=None), q=0, k=0, v=0) == 0
    assert "workspace" in P.lib.attn_status_str(-8).decode()


def test_the_norm_refuses():
    f = P.residual_rmsnorm_fwd_raw
    good = dict(x=OK, r=OK, w=OK, y=OK, s=OK, ro=OK, n=4, d=64, eps=1e-6, dt=0, fp8=1, g=128)
    call = lambda **x: f(*{**good, **x}.values(), 0)  # noqa: E731
    assert call(x=0) == -1 and call(y=0) == -1 and call(w=0) == -1 and call(ro=0) == -1 and call(s=0) == -1
    assert call(n=-1) == -2 and call(d=0) == -2 and call(d=(1 << 24) + 1) == -2 and call(g=64) == -2 and call(g=-128) == -2 and call(fp8=0) == -2
    assert call(dt=2) == -3 and call(eps=-1.0) == -4 and call(eps=float("nan")) == -4 and call(eps=float("inf")) == -4
    for name in "x r w y s ro".split():
        assert call(**{name: OK + 8}) == -6
    assert call(n=0, x=0, r=0, w=0, y=0, s=0, ro=0) == 0


@pytest.mark.parametrize("D", [32, 64, 128])
def test_a_key_s_place_in_a_page_of_any_size(L, D):
    """Pages of up to 2^30 keys are accepted: a key's place in one passes 32 bits."""
    L.key_offset.restype = ctypes.c_longlong
    for shift in range(31):
        size = 1 << shift
        for j in {0, 1, size // 2, size - 1, size, (1 << 23) - 1, 1 << 23, (1 << 23) + 77, 1 << 24, (1 << 30) - 1}:
            assert L.key_offset(j, size - 1, 2 * D) == j % size * 2 * D, (shift, j)


def test_hints_of_any_size(L):
    """max_q and max_kv are hints, any number that an int holds: work that is shared out fits 32 bits all the same, and more new tokens than there are
    count as all of them."""
    top = 2 ** 31 - 1
    r = random.Random(8)
    sizes = [(256, 256, 64, 8, 128), (1, 1, 8, 8, 64), (1 << 20, 1 << 20, 4, 4, 128), (1, 1 << 22, 64, 1, 128), (4096, 1 << 20, 128, 16, 64)]
    sizes += [(r.choice([1, 3, 64, 5000]), r.choice([1, 64, 4096, 100000]), 8 * r.choice([1, 4, 16]), r.choice([1, 2, 8]), r.choice([32, 64, 128])) for _ in range(300)]
    for B, T, Hq, Hk, D in sizes:
        for max_q in (1, T, top // 3, top):
            for max_kv in (0, 5000, 1 << 20, top - 1, top):
                p = plan(L, B, T, Hq, Hk, D, max_q, max_kv, 0)
                assert p == plan(L, B, T, Hq, Hk, D, min(max_q, T), max_kv, 0), (B, T, Hq, Hk, D, max_q, max_kv)
                assert 0 <= p["bytes"] == P.attn_paged_workspace(B, T, Hq, Hk, D, max_q, max_kv, 0)
                if p["balanced"]:
                    KB = 32 if p["rows"] < 128 and D == 128 else 64
                    tiles = B * -(-min(max_q, T) * (Hq // Hk) // p["rows"]) * Hk
                    assert tiles * (max_kv // KB + 9) < 2 ** 31, (B, T, Hq, Hk, D, max_q, max_kv)


def test_sizes_past_32_bits_have_no_workspace():
    good = [2, 3, 16, 8, 64, 2, 100000, 77]
    assert P.attn_paged_workspace(*good) > 0
    for i in range(8):
        for far in (2 ** 32, -2 ** 32, 2 ** 31, -2 ** 31 - 1):
            assert P.attn_paged_workspace(*good[:i], good[i] + far, *good[i + 1:]) == -1, (i, far)


def test_a_refusal_says_what_may_be_wrong_on_a_paged_cache():
    say = lambda status: P.lib.attn_status_str(status).decode()  # noqa: E731
    assert fwd(cache(page_size=24)) == -2 and "page_size a power of two" in say(-2)
    assert fwd(Hq=12) == -2 and "Hq a multiple of Hk" in say(-2) and append(rot=24) == -2 and "rot a multiple of 16" in say(-2)
    assert fwd(cache(kv_len=None)) == -1 and "kv_len" in say(-1) and append(cos=0) == -1 and "cos" in say(-1)
    assert fwd(lse=OK + 2) == -7 and fwd(lse=OK + 4) != -7 and "4-byte" in say(-7)
    # the limits that the header names: at them, and past them
    for at, past in ((dict(B=1 << 18, Hk=16, page_stride=1 << 20), dict(B=1 << 18, Hk=32, page_stride=1 << 20)), (dict(T=1 << 22), dict(T=(1 << 22) + 1)), (dict(width=1 << 26, table_stride=1 << 26), dict(width=(1 << 26) + 1, table_stride=1 << 27)),
                     (dict(n_pages=1 << 10, page_stride=1 << 30), dict(n_pages=1 << 10, page_stride=(1 << 30) + 8))):
        stop = dict(k=None)        # (a null pointer is found after the sizes: nothing is launched)
        assert append(cache(**at, **stop), q=0, Hq=0) == -1 and append(cache(**past, **stop), q=0, Hq=0) == -2, (at, past)
