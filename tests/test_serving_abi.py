"""What the serving calls refuse, and with which code, before anything reaches a GPU; their size query."""
import ctypes
import os

import pytest

from paper_2602_04163_amd import binding

P = 1 << 20                              # an aligned address that is never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2602_04163_amd import build
        build.build(verbose=False)
    return binding.load()


LINEAR = dict(planes=P, coefs=P, d_out=64, d_in=128, bits=2, group=32, X=P, n_tok=3, ldx=128, dtype=1, bias=None, act=0,
              residual=None, ldr=0, Y=P, ldy=64, ws=None, ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(planes=None), -1), (dict(planes=P + 2), -1), (dict(coefs=None), -2), (dict(coefs=P + 1), -2), (dict(d_out=0), -3),
    (dict(d_in=0), -4), (dict(d_in=100), -4), (dict(bits=0), -5), (dict(bits=5), -5), (dict(group=0), -6), (dict(group=48), -6),
    (dict(group=96), -6), (dict(X=None), -7), (dict(X=P + 1), -7), (dict(n_tok=-1), -8), (dict(ldx=127), -9), (dict(dtype=0), -10),
    (dict(dtype=3), -10), (dict(bias=P + 1), -11), (dict(act=-1), -12), (dict(act=5), -12), (dict(residual=P + 1), -13),
    (dict(residual=P, ldr=63), -14), (dict(Y=None), -15), (dict(Y=P + 1), -15), (dict(ldy=63), -16),
    (dict(n_tok=1000), -17), (dict(n_tok=1000, ws=P + 16, ws_bytes=1 << 30), -17), (dict(n_tok=1000, ws=P, ws_bytes=1000), -18),
    (dict(n_tok=0, X=None, Y=None), 0)])
def test_linear_refuses(lib, change, code):
    assert lib.bpdq_linear(*{**LINEAR, **change}.values()) == code


def test_linear_workspace(lib):
    size = lib.bpdq_linear_workspace_bytes
    assert size(0, 128) == size(1, 128) == size(-1, 128) == size(1000, 100) == size(1000, 0) == 0
    for n, d in ((33, 32), (1000, 4096), (4096, 18944), (70000, 29568)):
        assert size(n, d) % 256 == 0 and size(n, d) >= 2 * n * d
    assert size(1 << 20, 29568) > 1 << 35                # counted in more than 32 bits


def _cache(**change):
    f = {**dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=4, n_kv=2, page=64, head_dim=128), **change}
    return ctypes.byref(binding.BpdqKvCache(*f.values()))


BAD_CACHES = [dict(k=None), dict(k=P + 8), dict(v=None), dict(v=P + 8), dict(k_scale=None), dict(k_scale=P + 2), dict(v_scale=None),
              dict(n_pages=0), dict(n_kv=0), dict(page=0), dict(page=32), dict(page=96), dict(page=512), dict(head_dim=0),
              dict(head_dim=96), dict(head_dim=512)]

MOVE = dict(cache=None, table=P, max_pages=4, n_seq=2, pos=P, start=P, n_tok=9, max_tok=5, K=P, ldk=256, V=P, ldv=256, dtype=2,
            stream=None)


@pytest.mark.parametrize("name", ["bpdq_kv_write", "bpdq_kv_read"])
def test_the_cache_calls_refuse(lib, name):
    call = getattr(lib, name)
    for bad in BAD_CACHES:
        assert call(*{**MOVE, "cache": _cache(**bad)}.values()) == -1, bad
    assert call(*MOVE.values()) == -1
    for change, code in [(dict(table=None), -2), (dict(max_pages=0), -3), (dict(n_seq=-1), -4), (dict(n_seq=65536), -4),
                         (dict(pos=None), -5), (dict(start=None), -6), (dict(n_tok=-1), -7), (dict(max_tok=-1), -8),
                         (dict(K=None), -9), (dict(K=P + 1), -9), (dict(ldk=255), -10), (dict(V=None), -11), (dict(V=P + 1), -11),
                         (dict(ldv=255), -12), (dict(dtype=3), -13), (dict(dtype=-1), -13), (dict(dtype=0, K=P + 2), -9),
                         (dict(n_seq=0, table=None, pos=None), 0), (dict(n_tok=0, K=None, V=None), 0), (dict(max_tok=0, K=None), 0)]:
        assert call(*{**MOVE, "cache": _cache(), **change}.values()) == code, change


ATTENTION = dict(cache=None, table=P, max_pages=4, n_seq=2, kv_len=P, q_start=P, n_tok=9, max_q=5, max_kv=256, Q=P, ldq=1024, n_q=8,
                 dtype=1, scale=0.1, causal=1, window=0, out=P, ldo=1024, lse=None, ws=None, ws_bytes=0, stream=None)


def test_attention_refuses(lib):
    call = lib.bpdq_kv_attention
    for bad in BAD_CACHES:
        assert call(*{**ATTENTION, "cache": _cache(**bad)}.values()) == -1, bad
    for change, code in [(dict(table=None), -2), (dict(max_pages=0), -3), (dict(n_seq=-1), -4), (dict(n_seq=65536), -4),
                         (dict(kv_len=None), -5), (dict(q_start=None), -6), (dict(n_tok=-1), -7), (dict(max_q=-1), -8),
                         (dict(max_q=1 << 24), -8), (dict(max_kv=-1), -9), (dict(max_kv=257), -9), (dict(Q=None), -10),
                         (dict(Q=P + 1), -10), (dict(ldq=1023), -11), (dict(n_q=0), -12), (dict(n_q=7), -12), (dict(dtype=0), -13),
                         (dict(dtype=3), -13), (dict(scale=float("nan")), -14), (dict(scale=float("inf")), -14), (dict(window=-1), -16),
                         (dict(out=None), -17), (dict(out=P + 1), -17), (dict(ldo=1023), -18),
                         (dict(n_seq=0, table=None), 0), (dict(n_tok=0, Q=None), 0), (dict(max_q=0, Q=None), 0)]:
        assert call(*{**ATTENTION, "cache": _cache(), **change}.values()) == code, change


def test_a_split_call_wants_its_workspace(lib):
    need = lib.bpdq_kv_attention_workspace_bytes(1, 1, 65536, 8, 2, 128, 0)
    assert need > 0
    long = {**ATTENTION, "cache": _cache(n_pages=1024), "max_pages": 1024, "n_seq": 1, "max_q": 1, "max_kv": 65536, "n_tok": 1}
    assert lib.bpdq_kv_attention(*long.values()) == -20
    assert lib.bpdq_kv_attention(*{**long, "ws": P + 16, "ws_bytes": need}.values()) == -20
    assert lib.bpdq_kv_attention(*{**long, "ws": P, "ws_bytes": need - 1}.values()) == -21
    assert lib.bpdq_kv_attention_workspace_bytes(1, 1, 64, 8, 2, 128, 0) == 0          # one tile: nothing to split
    assert lib.bpdq_kv_attention_workspace_bytes(1, 1, 65536, 8, 2, 128, 64) == 0      # nor inside a short window
    for bad in [(0, 1, 64, 8, 2, 128, 0), (1, 0, 64, 8, 2, 128, 0), (1, 1, 0, 8, 2, 128, 0), (1, 1, 65536, 7, 2, 128, 0),
                (1, 1, 65536, 8, 2, 96, 0), (1, 1, 65536, 8, 2, 128, -1), (1, 1, 65536, 8, 0, 128, 0)]:
        assert lib.bpdq_kv_attention_workspace_bytes(*bad) == 0


def test_attention_counts_positions_in_32_bits(lib):
    """Positions less a window, and the end of the last tile, have to stay within an int: caches end at 2^30 tokens."""
    wide = {**ATTENTION, "cache": _cache(), "max_pages": 1 << 25, "n_tok": 0}
    for most, code in [(1 << 30, 0), ((1 << 30) + 1, -9), ((1 << 31) - 1, -9)]:
        for window in (0, 16, most - 1):
            assert lib.bpdq_kv_attention(*{**wide, "max_kv": most, "window": window}.values()) == code, (most, window)
    size = lib.bpdq_kv_attention_workspace_bytes
    assert size(1, 1, 1 << 30, 8, 2, 128, 0) > 0 and size(1, 1, (1 << 30) + 1, 8, 2, 128, 0) == 0
