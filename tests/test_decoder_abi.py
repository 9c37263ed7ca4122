"""What the norm, rotary positions, the gated product and sampling refuse, and with which code, before anything reaches a GPU; the host's
frequencies against the oracle."""
import ctypes
import os

import numpy as np
import pytest

from oracle import decoder_oracle as do
from paper_2602_04163_amd import binding

P = 1 << 20                              # an aligned address that is never followed
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2602_04163_amd import build
        build.build(verbose=False)
    return binding.load()


GATED = dict(planes=P, coefs=P, d_out=64, d_in=128, bits=2, group=32, X=P, n_tok=3, ldx=128, dtype=1, bias=None, act=4, Y=P, ldy=64, ws=None,
             ws_bytes=0, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(planes=None), -1), (dict(planes=P + 2), -1), (dict(coefs=None), -2), (dict(coefs=P + 1), -2), (dict(d_out=0), -3),
    (dict(d_out=-1), -3), (dict(d_out=(1 << 31) - 1), -3), (dict(d_out=1 << 27, d_in=128), -3), (dict(d_in=0), -4), (dict(d_in=100), -4),
    (dict(bits=0), -5), (dict(bits=5), -5), (dict(group=0), -6), (dict(group=48), -6), (dict(group=96), -6), (dict(X=None), -7),
    (dict(X=P + 1), -7), (dict(n_tok=-1), -8), (dict(ldx=127), -9), (dict(dtype=0), -10), (dict(dtype=3), -10), (dict(bias=P + 1), -11),
    (dict(act=-1), -12), (dict(act=5), -12), (dict(Y=None), -13), (dict(Y=P + 1), -13), (dict(ldy=63), -14), (dict(n_tok=1000), -15),
    (dict(n_tok=1000, ws=P + 16, ws_bytes=1 << 30), -15), (dict(n_tok=1000, ws=P, ws_bytes=1000), -16),
    (dict(n_tok=0, X=None, Y=None), 0)])
def test_gated_refuses(lib, change, code):
    assert lib.bpdq_gated_linear(*{**GATED, **change}.values()) == code


NORM = dict(X=P, n_tok=3, d=64, ldx=64, dtype=2, residual=None, ldr=0, rdtype=2, S=None, lds=0, weight=P, offset=0.0, eps=1e-6)
WITH = dict(residual=P, ldr=64, S=P, lds=64)


@pytest.mark.parametrize("change,code", [
    (dict(X=None), -1), (dict(X=P + 1), -1), (dict(dtype=0, X=P + 2), -1), (dict(n_tok=-1), -2), (dict(d=0), -3), (dict(d=65537), -3),
    (dict(ldx=63), -4), (dict(dtype=3), -5), (dict(dtype=-1), -5), (dict(residual=P + 1, ldr=64), -6), (dict(residual=P, ldr=63), -7),
    (dict(residual=P, ldr=64, rdtype=1), -8), (dict(residual=P + 2, ldr=64, rdtype=0), -6), (dict(S=P, lds=64), -9), ({**WITH, "S": P + 1}, -9),
    ({**WITH, "lds": 63}, -10), (dict(weight=P + 1), -11), (dict(offset=NAN), -12), (dict(offset=INF), -12), (dict(eps=0.0), -13),
    (dict(eps=-1.0), -13), (dict(eps=NAN), -13), (dict(eps=INF), -13), (dict(eps=1e-39), -13), (dict(n_tok=0, X=None), 0)])
def test_norms_refuse(lib, change, code):
    plain = {**NORM, **change, "Y": P, "ldy": 64, "stream": None}
    assert lib.bpdq_rms_norm(*plain.values()) == code
    q8 = {**NORM, **change, "group": 0, "codes": P, "ldc": 64, "scales": P, "stream": None}
    assert lib.bpdq_rms_norm_q8(*q8.values()) == code


def test_norms_count_their_threads(lib):
    """A grid ends at 2^32 threads: rows of 8192 values take 512 each, of 32 four."""
    most = (1 << 31) - 1
    plain = {**NORM, "Y": P, "ldy": 1 << 16, "stream": None, "n_tok": most, "d": 8192, "ldx": 8192}
    assert lib.bpdq_rms_norm(*plain.values()) == -2


def test_norms_refuse_outputs(lib):
    plain = {**NORM, "Y": P, "ldy": 64, "stream": None}
    for change, code in [(dict(Y=None), -14), (dict(Y=P + 1), -14), (dict(ldy=63), -15)]:
        assert lib.bpdq_rms_norm(*{**plain, **change}.values()) == code
    q8 = {**NORM, "group": 0, "codes": P, "ldc": 64, "scales": P, "stream": None}
    for change, code in [(dict(group=-32), -14), (dict(group=48), -14), (dict(group=128), -14), (dict(group=8), -14),
                         (dict(group=512, d=512, ldx=512, ldc=512), -14), (dict(codes=None), -15), (dict(ldc=63), -16),
                         (dict(scales=None), -17), (dict(scales=P + 2), -17), (dict(group=48, n_tok=0), -14)]:
        assert lib.bpdq_rms_norm_q8(*{**q8, **change}.values()) == code


ROTARY = dict(freq=P, rot=64, layout=0, mscale=1.0, inverse=0, pos=P, start=P, n_seq=2, n_tok=9, max_tok=5, Q=P, ldq=512, n_q=8, K=P, ldk=128,
              n_kv=2, head_dim=64, dtype=2, Q_out=P, ldqo=512, K_out=P, ldko=128, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(freq=None), -1), (dict(freq=P + 4), -1), (dict(rot=0), -2), (dict(rot=63), -2), (dict(rot=66), -2), (dict(rot=-2), -2),
    (dict(layout=2), -3), (dict(layout=-1), -3), (dict(mscale=NAN), -4), (dict(mscale=INF), -4), (dict(pos=None), -6), (dict(pos=P + 1), -6),
    (dict(start=None), -7), (dict(start=P + 2), -7), (dict(n_seq=-1), -8), (dict(n_seq=65536), -8), (dict(n_tok=-1), -9),
    (dict(max_tok=-1), -10), (dict(Q=None), -11), (dict(Q=P + 1), -11), (dict(dtype=0, Q=P + 2), -11), (dict(ldq=511), -12), (dict(n_q=-1), -13),
    (dict(n_q=65536), -13), (dict(K=None), -14), (dict(K=P + 1), -14), (dict(ldk=127), -15), (dict(n_kv=-1), -16), (dict(head_dim=0), -17),
    (dict(head_dim=514), -17), (dict(dtype=3), -18), (dict(Q_out=None), -19), (dict(Q_out=P + 1), -19), (dict(ldqo=511), -20),
    (dict(ldqo=520), -20), (dict(K_out=None), -21), (dict(ldko=127), -22), (dict(ldko=136), -22),
    (dict(n_seq=0, pos=None), 0), (dict(n_tok=0, Q=None), 0), (dict(max_tok=0, Q=None), 0), (dict(n_q=0, n_kv=0, Q=None, K=None), 0)])
def test_rotary_refuses(lib, change, code):
    assert lib.bpdq_rotary(*{**ROTARY, **change}.values()) == code


@pytest.mark.parametrize("rot,base,scaling,factor,low,high,original", [
    (128, 1e6, "plain", 1.0, 1.0, 32.0, 0), (64, 1e4, "linear", 4.0, 1.0, 32.0, 0), (128, 1e4, "ntk", 8.0, 1.0, 32.0, 0),
    (128, 1e6, "yarn", 4.0, 1.0, 32.0, 32768), (32, 1e4, "yarn", 40.0, 1.0, 32.0, 4096), (2, 1e4, "yarn", 4.0, 1.0, 32.0, 4096),
    (64, 5e5, "yarn", 2.0, 1.0, 32.0, 8), (128, 5e5, "bands", 8.0, 1.0, 4.0, 8192), (6, 1e4, "bands", 32.0, 0.5, 64.0, 131072)])
def test_frequencies(lib, rot, base, scaling, factor, low, high, original):
    freq, mscale = binding.bpdq_rotary_frequencies(rot, base, scaling, factor, low, high, original)
    want, m = do.rotary_frequencies(rot, base, scaling, factor, low, high, original)
    # powers and logarithms of libm and Python, a few units in the last place of 2^-52 on exponents up to log2(1e6)
    assert np.allclose(freq.numpy(), want, rtol=1e-13, atol=0.0) and abs(mscale - m) < 1e-14


def test_frequencies_refuse(lib):
    ok = dict(rot=8, base=1e4, scaling=3, factor=4.0, low=1.0, high=32.0, original=4096, freq=(ctypes.c_double * 4)(), mscale=None)
    args = {**ok, "freq": ctypes.addressof(ok["freq"])}
    assert lib.bpdq_rotary_frequencies(*args.values()) == 0
    for change, code in [(dict(rot=0), -1), (dict(rot=7), -1), (dict(rot=2, scaling=2), -1), (dict(base=1.0), -2), (dict(base=NAN), -2),
                         (dict(scaling=5), -3), (dict(scaling=-1), -3), (dict(factor=0.5), -4), (dict(factor=NAN), -4), (dict(low=0.0), -5),
                         (dict(high=1.0), -6), (dict(high=INF), -6), (dict(original=0), -7), (dict(freq=None), -8)]:
        assert lib.bpdq_rotary_frequencies(*{**args, **change}.values()) == code
    with pytest.raises(binding.BpdqError, match="scaling"):
        binding.bpdq_rotary_frequencies(8, scaling="none")
    with pytest.raises(binding.BpdqError, match="argument 1"):
        binding.bpdq_rotary_frequencies(-2)


SAMPLE = dict(logits=P, n_tok=3, n_vocab=1000, ldl=1000, dtype=2, temperature=P, top_k=P, top_p=P, min_p=P, u=P, token=P, prob=P, ws=P,
              ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(logits=None), -1), (dict(logits=P + 1), -1), (dict(logits=P + 2, dtype=0), -1), (dict(n_tok=-1), -2), (dict(n_tok=(1 << 15) + 1), -2), (dict(n_vocab=0), -3),
    (dict(n_vocab=(1 << 20) + 1), -3), (dict(ldl=999), -4), (dict(dtype=3), -5), (dict(dtype=-1), -5), (dict(temperature=P + 2), -6),
    (dict(top_k=P + 1), -7), (dict(top_p=P + 2), -8), (dict(min_p=P + 3), -9), (dict(u=None), -10), (dict(u=P + 2), -10), (dict(token=None), -11),
    (dict(token=P + 1), -11), (dict(prob=P + 2), -12), (dict(n_tok=0, logits=None, u=None, token=None, ws=None, ws_bytes=0), 0)])
def test_sample_refuses(lib, change, code):
    assert lib.bpdq_sample(*{**SAMPLE, **change}.values()) == code


def test_sample_wants_its_workspace(lib):
    size = lib.bpdq_sample_workspace_bytes
    assert size(0, 1000) == size(-1, 1000) == size(3, 0) == size(3, (1 << 20) + 1) == 0
    need = size(3, 1000)
    if need:
        assert lib.bpdq_sample(*{**SAMPLE, "ws": None}.values()) == -13
        assert lib.bpdq_sample(*{**SAMPLE, "ws": P + 64}.values()) == -13
        assert lib.bpdq_sample(*{**SAMPLE, "ws_bytes": need - 1}.values()) == -14
    assert size(1 << 15, 1 << 20) > size(1 << 10, 1 << 20) > 0 and size((1 << 15) + 1, 1000) == 0
