"""What the binding of the serving calls refuses of tensors before a pointer leaves it.  The tensors here lie on the host and only say that
they are on a GPU: a call that got past its checks would stop at the stand-in for the library."""
import pytest
import torch

from paper_2602_04163_amd import binding as bq


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(t):
    return t.as_subclass(OnGpu)


class Reached(Exception):
    pass


class Library:
    """In the library's place: its size queries ask for nothing, its calls say that they were reached."""

    def __getattr__(self, name):
        if name.endswith("_workspace_bytes"):
            return lambda *a: 0
        raise Reached(name)


@pytest.fixture
def stand_in(monkeypatch):
    monkeypatch.setattr(bq, "_lib", Library())


N, D_IN, D_OUT, KV, DIM = 5, 64, 32, 2, 64


def _linear(X=None, residual=None, Y=None):
    half = torch.float16
    return bq.bpdq_linear(gpu(torch.zeros((2, D_OUT, D_IN // 32), dtype=torch.int32)), gpu(torch.zeros((3, D_OUT, 2), dtype=half)), 32,
                          gpu(torch.zeros((N, D_IN), dtype=half)) if X is None else X, residual=residual,
                          Y=gpu(torch.zeros((N, D_OUT), dtype=half)) if Y is None else Y)


def _ints(n):
    return gpu(torch.zeros(n, dtype=torch.int32))


def _cache():
    codes, scale = torch.zeros((1, KV, 64, DIM), dtype=torch.uint8), torch.zeros((1, KV))
    return bq.KvCache(gpu(codes), gpu(codes.clone()), gpu(scale), gpu(scale.clone()))


def _tokens(heads=KV):
    return gpu(torch.zeros((N, heads, DIM), dtype=torch.float16))


def _write(K=None, V=None):
    bq.bpdq_kv_write(_cache(), _ints((1, 1)), _ints(1), _ints(2), _tokens() if K is None else K, _tokens() if V is None else V)


def _read(K=None, V=None):
    bq.bpdq_kv_read(_cache(), _ints((1, 1)), _ints(1), _ints(2), N, dtype=torch.float16, K=_tokens() if K is None else K,
                    V=_tokens() if V is None else V)


def _attend(Q=None, out=None):
    bq.bpdq_kv_attention(_cache(), _ints((1, 1)), _ints(1), _ints(2), _tokens(4) if Q is None else Q,
                         out=_tokens(4) if out is None else out)


# the calls' tensors of rows: the call, the argument, the shape of a row
ROWS = [(_linear, "X", (D_IN,)), (_linear, "residual", (D_OUT,)), (_linear, "Y", (D_OUT,)), (_write, "K", (KV, DIM)),
        (_write, "V", (KV, DIM)), (_read, "K", (KV, DIM)), (_read, "V", (KV, DIM)), (_attend, "Q", (4, DIM)), (_attend, "out", (4, DIM))]


def _with_row_stride(shape, stride, n=N):
    size = torch.Size(shape).numel()
    inner = (shape[1], 1) if len(shape) == 2 else (1,)
    return gpu(torch.zeros(n * (size + stride) + size, dtype=torch.float16).as_strided((n, *shape), (stride, *inner)))


@pytest.mark.parametrize("call,name,shape", ROWS)
def test_rows_that_overlap_are_refused(stand_in, call, name, shape):
    """A row stride below a row's length, 0 (one row shown n times) among them: taken as dense, such a tensor would be read or written
    behind its end."""
    size = torch.Size(shape).numel()
    for stride in (0, 1, 8, size // 2, size - 1):
        with pytest.raises(bq.BpdqError, match=name):
            call(**{name: _with_row_stride(shape, stride)})
    with pytest.raises(bq.BpdqError, match=name):
        call(**{name: gpu(torch.zeros((1, *shape), dtype=torch.float16)).expand(N, *shape)})
    for stride in (size, size + 1, 3 * size):
        with pytest.raises(Reached):
            call(**{name: _with_row_stride(shape, stride)})


def test_the_stride_of_a_single_row_says_nothing():
    for stride in (0, 1, D_IN, 5 * D_IN):
        assert bq._rows(_with_row_stride((D_IN,), stride, 1), torch.float16, (1, D_IN), "X") == D_IN
    assert bq._rows(_with_row_stride((D_IN,), 5 * D_IN), torch.float16, (N, D_IN), "X") == 5 * D_IN
    assert bq._rows(_with_row_stride((D_IN,), D_IN, 0), torch.float16, (0, D_IN), "X") == D_IN


def _linear_ws(ws):
    bq.bpdq_linear(gpu(torch.zeros((2, D_OUT, 2), dtype=torch.int32)), gpu(torch.zeros((3, D_OUT, 2), dtype=torch.float16)), 32,
                   gpu(torch.zeros((N, D_IN), dtype=torch.float16)), Y=gpu(torch.zeros((N, D_OUT), dtype=torch.float16)), ws=ws)


def _attend_ws(ws):
    bq.bpdq_kv_attention(_cache(), _ints((1, 1)), _ints(1), _ints(2), _tokens(4), out=_tokens(4), ws=ws)


def _square():
    return gpu(torch.zeros((64, 64)))


WITH_WS = {"linear": _linear_ws, "attention": _attend_ws, "prepare": lambda ws: bq.bpdq_prepare(_square(), U=_square(), ws=ws),
           "hessian": lambda ws: bq.bpdq_hessian_accumulate(_square(), _square(), ws=ws),
           "layer": lambda ws: bq.bpdq_quantize_layer(_square(), _square(), None, bq.make_params(2, 64, 64, 1), ws=ws),
           "layers": lambda ws: bq.bpdq_quantize_layers(_square(), [32, 64], _square(), None, bq.make_params(2, 64, 64, 1), ws=ws)}


@pytest.mark.parametrize("name", list(WITH_WS))
def test_a_workspace_lies_on_the_gpu_in_one_piece(monkeypatch, name):
    """On the host, or with gaps, a caller's workspace is refused; of whatever type, it counts by its bytes."""
    seen = []

    class Calls:
        def __getattr__(self, entry):
            return (lambda *a: 0) if entry.endswith("_workspace_bytes") else lambda *a: seen.append(a) or 0

    monkeypatch.setattr(bq, "_lib", Calls())
    monkeypatch.setattr(bq, "_stream", lambda: None)
    for bad in (torch.zeros(4096, dtype=torch.uint8), gpu(torch.zeros(4096, dtype=torch.uint8))[::2],
                gpu(torch.zeros((64, 64), dtype=torch.uint8)).t()):
        with pytest.raises(bq.BpdqError, match="ws"):
            WITH_WS[name](bad)
    assert not seen
    for t in (torch.uint8, torch.float32, torch.float64):
        ws = gpu(torch.zeros(500, dtype=t))
        WITH_WS[name](ws)
        at = seen[-1].index(ws.data_ptr())
        assert seen[-1][at + 1] == 500 * ws.element_size()
