"""What the binding of the norm, rotary positions, the gated product and sampling refuses of tensors before a pointer leaves it.  The tensors
here lie on the host and only say that they are on a GPU: a call that got past its checks would stop at the stand-in for the library."""
import pytest
import torch

from paper_2602_04163_amd import binding as bq

from test_serving_binding import Library, Reached, gpu

N, D, F, Q, KV, DIM, V = 5, 64, 32, 4, 2, 16, 100
HALF, WIDE, INT = torch.float16, torch.float32, torch.int32


@pytest.fixture(autouse=True)
def stand_in(monkeypatch):
    monkeypatch.setattr(bq, "_lib", Library())
    monkeypatch.setattr(bq, "_here", lambda *tensors: None)
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, empty=torch.empty, **kw: gpu(empty(*a, **kw)))
    monkeypatch.setattr(bq, "_like", lambda t: gpu(torch.zeros(t.shape, dtype=t.dtype)))


def of(*shape, dtype=HALF):
    return gpu(torch.zeros(shape, dtype=dtype))


def norm(X=None, weight=None, residual=None, **kw):
    bq.bpdq_rms_norm(of(N, D) if X is None else X, of(D) if weight is None else weight, residual=residual, **kw)


def norm_q8(X=None, **kw):
    bq.bpdq_rms_norm_q8(of(N, D) if X is None else X, **kw)


def rotary(freq=None, pos=None, tok_start=None, Q_=None, K=None, **kw):
    bq.bpdq_rotary(of(DIM // 2, dtype=torch.float64) if freq is None else freq, of(2, dtype=INT) if pos is None else pos,
                   of(3, dtype=INT) if tok_start is None else tok_start, of(N, Q, DIM) if Q_ is None else Q_,
                   of(N, KV, DIM) if K is None else K, **kw)


def gated(planes=None, coefs=None, X=None, group=32, **kw):
    bq.bpdq_gated_linear(of(2, 2 * F, D // 32, dtype=INT) if planes is None else planes, of(3, 2 * F, 2) if coefs is None else coefs, group,
                         of(N, D) if X is None else X, **kw)


def sample(logits=None, u=None, **kw):
    bq.bpdq_sample(of(N, V) if logits is None else logits, of(N, dtype=WIDE) if u is None else u, **kw)


HOST = torch.zeros((N, D), dtype=HALF)


@pytest.mark.parametrize("call,kw,name", [
    (norm, dict(X=HOST), "X"), (norm, dict(X=of(N, D, dtype=torch.float64)), "X"), (norm, dict(X=of(N, D, 1)), "X"),
    (norm, dict(X=of(D, N).t()), "X"), (norm, dict(X=of(1, D).expand(N, D)), "X"), (norm, dict(weight=of(D + 1)), "weight"),
    (norm, dict(weight=of(D, dtype=WIDE)), "weight"), (norm, dict(weight=of(2 * D)[::2]), "weight"), (norm, dict(residual=of(N + 1, D)), "residual"),
    (norm, dict(residual=of(N, D, dtype=torch.bfloat16)), "residual"), (norm, dict(S=of(N, D)), "S"),
    (norm, dict(residual=of(N, D, dtype=WIDE), S=of(N, D)), "S"), (norm, dict(Y=of(N, D, dtype=WIDE)), "Y"), (norm, dict(Y=of(N, D + 1)), "Y"),
    (norm_q8, dict(codes=of(N, D, dtype=torch.uint8)), "codes"), (norm_q8, dict(scales=of(N, 2, dtype=WIDE)), "scales"),
    (norm_q8, dict(group=32, scales=of(N, 1, dtype=WIDE)), "scales"), (norm_q8, dict(scales=of(N, 1)), "scales"),
    (rotary, dict(freq=of(DIM // 2, dtype=WIDE)), "freq"), (rotary, dict(pos=of(2, dtype=torch.int64)), "pos"),
    (rotary, dict(tok_start=of(2, dtype=INT)), "tok_start"), (rotary, dict(Q_=of(N, Q * DIM)), "Q"), (rotary, dict(Q_=of(N, Q, DIM, dtype=torch.float64)), "Q"),
    (rotary, dict(Q_=of(Q, N, DIM).transpose(0, 1)), "Q"), (rotary, dict(K=of(N + 1, KV, DIM)), "K"), (rotary, dict(K=of(N, KV, DIM + 2)), "K"),
    (rotary, dict(K=of(N, KV, DIM, dtype=WIDE)), "K"), (rotary, dict(Q_out=of(N, Q, DIM, dtype=WIDE)), "Q_out"),
    (rotary, dict(K_out=of(N, Q, DIM)), "K_out"), (rotary, dict(layout="neox"), "layout"),
    (gated, dict(planes=of(2, 2 * F + 1, 2, dtype=INT)), "planes"), (gated, dict(coefs=of(3, F, 2)), "coefs_h"), (gated, dict(group=0), "coefs_h"),
    (gated, dict(X=of(N, D, dtype=WIDE)), "X"), (gated, dict(X=of(N, D + 32)), "X"), (gated, dict(act="tanh"), "act"),
    (gated, dict(bias=of(F)), "bias"), (gated, dict(bias=of(2 * F, dtype=WIDE)), "bias"), (gated, dict(Y=of(N, 2 * F)), "Y"),
    (sample, dict(logits=of(N, V, dtype=torch.float64)), "logits"), (sample, dict(logits=of(N, 1, V)), "logits"), (sample, dict(u=of(N + 1, dtype=WIDE)), "u"),
    (sample, dict(u=of(N)), "u"), (sample, dict(temperature=of(N)), "temperature"), (sample, dict(top_k=of(N, dtype=torch.int64)), "top_k"),
    (sample, dict(top_p=of(2 * N, dtype=WIDE)[::2]), "top_p"), (sample, dict(min_p=torch.zeros(N)), "min_p"),
    (sample, dict(token=of(N, dtype=torch.int64)), "token"), (sample, dict(prob=of(N)), "prob")])
def test_tensors_are_refused(call, kw, name):
    with pytest.raises(bq.BpdqError, match=name):
        call(**kw)


@pytest.mark.parametrize("call,kw", [
    (norm, {}), (norm, dict(residual=of(N, D), S=of(N, D))), (norm, dict(residual=of(N, D, dtype=WIDE))), (norm_q8, dict(group=32)), (rotary, {}),
    (rotary, dict(Q_=of(N, (Q + 2 * KV) * DIM)[:, :Q * DIM].unflatten(1, (Q, DIM)))), (gated, {}), (gated, dict(bias=of(2 * F))),
    (sample, {}), (sample, dict(want_prob=True)), (sample, dict(logits=of(N, 2 * V)[:, :V], top_k=of(N, dtype=INT)))])
def test_what_is_taken_reaches_the_library(call, kw):
    with pytest.raises(Reached):
        call(**kw)


@pytest.mark.parametrize("call", [gated, sample])
def test_a_workspace_lies_on_the_gpu_in_one_piece(monkeypatch, call):
    seen = []

    class Calls:
        def __getattr__(self, entry):
            return (lambda *a: 0) if entry.endswith("_workspace_bytes") else lambda *a: seen.append(a) or 0

    monkeypatch.setattr(bq, "_lib", Calls())
    monkeypatch.setattr(bq, "_stream", lambda: None)
    for bad in (torch.zeros(4096, dtype=torch.uint8), of(4096)[::2], of(64, 64).t()):
        with pytest.raises(bq.BpdqError, match="ws"):
            call(ws=bad)
    assert not seen
    ws = of(500, dtype=torch.float64)
    call(ws=ws)
    assert seen[-1][seen[-1].index(ws.data_ptr()) + 1] == 4000


def test_q_alone():
    with pytest.raises(Reached):
        bq.bpdq_rotary(of(8, dtype=torch.float64), of(1, dtype=INT), of(2, dtype=INT), of(N, Q, DIM))
    with pytest.raises(bq.BpdqError, match="K_out"):
        bq.bpdq_rotary(of(8, dtype=torch.float64), of(1, dtype=INT), of(2, dtype=INT), of(N, Q, DIM), K_out=of(N, KV, DIM))


def test_another_gpu_is_refused(monkeypatch):
    monkeypatch.undo()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)

    class There:
        def get_device(self):
            return 0

    with pytest.raises(bq.BpdqError, match="GPU 0"):
        bq._here(None, There())
