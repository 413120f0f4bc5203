"""The training step's calls over the recording runtime, without a GPU: what they refuse, and what becomes of their scratch."""
import pytest

import host_calls

_CALLS = r'''
import math
INVALID, STATE = 1, 5
F32, BF16, F16 = 0, 1, 2
f32 = ctypes.c_float
lib.rg_mx4_row_words.restype = i64
class Tensor(Structure):
    _fields_ = [("in_", p), ("out", p), ("size", i64), ("type", i32)]
c = context()
def message(): return lib.rg_last_error(c).decode()
def quantize(x=None, type=F32, x_stride=100, n=10, n_dev=0, dim=100, packed=None, packed_stride=20, stream=0):
    return lib.rg_mx4_quantize(c, p(address() if x is None else x), i32(type), i64(x_stride), i64(n), p(n_dev), i32(dim),
                               p(address() if packed is None else packed), i64(packed_stride), p(stream))
def dequantize(packed=None, packed_stride=20, n=10, n_dev=0, dim=100, x=None, type=F32, x_stride=100, stream=0):
    return lib.rg_mx4_dequantize(c, p(address() if packed is None else packed), i64(packed_stride), i64(n), p(n_dev), i32(dim),
                                 p(address() if x is None else x), i32(type), i64(x_stride), p(stream))
def matmul(rows=None, rows_stride=20, n=10, n_dev=0, weight=None, weight_stride=20, out_dim=30, dim=100, y=None, type=F32, y_stride=30, stream=0):
    return lib.rg_mx4_matmul(c, p(address() if rows is None else rows), i64(rows_stride), i64(n), p(n_dev), p(address() if weight is None else weight),
                             i64(weight_stride), i32(out_dim), i32(dim), p(address() if y is None else y), i32(type), i64(y_stride), p(stream))
def matmul_grad(dy=None, type=F32, dy_stride=30, rows=None, rows_stride=20, n=10, n_dev=0, out_dim=30, dim=100, grad=None, grad_stride=100, stream=0):
    return lib.rg_mx4_matmul_grad(c, p(address() if dy is None else dy), i32(type), i64(dy_stride), p(address() if rows is None else rows),
                                  i64(rows_stride), i64(n), p(n_dev), i32(out_dim), i32(dim), p(address() if grad is None else grad),
                                  i64(grad_stride), p(stream))
def norm(x=None, type=F32, x_stride=100, n=10, n_dev=0, dim=100, gamma=0, beta=0, eps=1e-5, y=None, y_stride=100, mean=0, rstd=0, stream=0):
    return lib.rg_layer_norm(c, p(address() if x is None else x), i32(type), i64(x_stride), i64(n), p(n_dev), i32(dim), p(gamma), p(beta), f32(eps),
                             p(address() if y is None else y), i64(y_stride), p(mean), p(rstd), p(stream))
def norm_grad(dy=None, dy_stride=100, x=None, x_stride=100, type=F32, n=10, n_dev=0, dim=100, gamma=0, mean=None, rstd=None, dx=None,
              dx_stride=100, dgamma=None, dbeta=None, stream=0):
    a = lambda v: p(address() if v is None else v)
    return lib.rg_layer_norm_grad(c, a(dy), i64(dy_stride), a(x), i64(x_stride), i32(type), i64(n), p(n_dev), i32(dim), p(gamma), a(mean), a(rstd),
                                  a(dx), i64(dx_stride), a(dgamma), a(dbeta), p(stream))
def clip(sizes=(5, 7), types=None, max_norm=1.0, norm=None, ins=None, outs=None, count=None, stream=0):
    t = (Tensor * max(len(sizes), 1))()
    for i, k in enumerate(sizes):
        t[i] = Tensor(address() if ins is None else ins[i], address() if outs is None else outs[i], k, F32 if types is None else types[i])
    return lib.rg_clip_grad_norm(c, t, i32(len(sizes) if count is None else count), f32(max_norm), p(address() if norm is None else norm), p(stream))
def refuses(status, text):
    assert status == INVALID and text in message(), (status, message())
    assert not kernels()
'''


def run(program):
    return host_calls.run(_CALLS + program)


def test_packed_calls_refuse():
    run(r'''
assert [lib.rg_mx4_row_words(i32(d)) for d in (0, -1, 1, 32, 33, 100, 256, 602, 65536, 65537)] == [0, 0, 5, 5, 9, 17, 34, 81, 8704, 0]
for call, name in ((quantize, "rg_mx4_quantize"), (dequantize, "rg_mx4_dequantize")):
    refuses(call(n=-1), name)
    refuses(call(n=1 << 31), "out of range")
    refuses(call(dim=0), "dim")
    refuses(call(dim=65537, x_stride=70000, packed_stride=70000), "dim")
    refuses(call(type=3), "type")
    refuses(call(x_stride=99), "stride")
    refuses(call(packed_stride=16), "stride")
    refuses(call(x=0), "null")
    refuses(call(packed=0), "null")
    refuses(call(x=0x5002), "aligned")
    refuses(call(x=0x5001, type=BF16), "aligned")
    refuses(call(packed=0x5002), "aligned")
    assert call(x=0x5002, type=F16) == OK and call(n=0, x=0, packed=0) == OK and len(kernels()) == 1
    assert lib.rg_mx4_quantize(None, None, 0, i64(0), i64(0), None, 0, None, i64(0), None) == INVALID
''')


def test_products_refuse():
    run(r'''
for call in (matmul, matmul_grad):
    refuses(call(n=-1), "out of range")
    refuses(call(dim=0), "dim")
    refuses(call(out_dim=0), "out_dim")
    refuses(call(out_dim=65537), "out_dim")
    refuses(call(type=-1), "type")
    refuses(call(rows_stride=16), "stride")
    refuses(call(rows=0), "null")
    refuses(call(rows=0x7001), "aligned")
refuses(matmul(weight_stride=16), "stride")
refuses(matmul(y_stride=29), "stride")
refuses(matmul(weight=0), "null")
refuses(matmul(y=0), "null")
refuses(matmul(y=0x7001, type=F16), "aligned")
refuses(matmul_grad(dy_stride=29), "stride")
refuses(matmul_grad(grad_stride=99), "stride")
refuses(matmul_grad(dy=0), "null")
refuses(matmul_grad(grad=0), "null")
refuses(matmul_grad(n=0, grad=0), "null")
assert matmul(n=0, rows=0, weight=0, y=0) == OK and not kernels()
assert matmul_grad(n=0, rows=0, dy=0) == OK and len(kernels()) >= 1      # zeros
''')


def test_norms_refuse():
    run(r'''
for call in (norm, norm_grad):
    refuses(call(n=-1), "out of range")
    refuses(call(dim=0), "dim")
    refuses(call(dim=65537, x_stride=70000), "dim")
    refuses(call(type=9), "type")
    refuses(call(x_stride=99), "stride")
    refuses(call(x=0), "null")
    refuses(call(x=0x7001, type=BF16), "aligned")
    refuses(call(gamma=0x7002), "aligned")
for eps in (-1e-9, math.nan):
    refuses(norm(eps=eps), "eps")
refuses(norm(y=0), "null")
refuses(norm(y_stride=99), "stride")
refuses(norm(x=0x8000, y=0x8000, x_stride=100, y_stride=104), "stride")
refuses(norm_grad(dy_stride=99), "stride")
refuses(norm_grad(dx_stride=99), "stride")
refuses(norm_grad(dy=0), "null")
refuses(norm_grad(mean=0), "null")
refuses(norm_grad(rstd=0), "null")
refuses(norm_grad(dx=0x8000, dy=0x8000, dx_stride=104), "stride")
assert norm(n=0, x=0, y=0) == OK and norm_grad(dx=0, dx_stride=0, dgamma=0, dbeta=0) == OK and not kernels()
assert norm_grad(n=0, x=0, dy=0, mean=0, rstd=0, dx=0, dx_stride=0) == OK and len(kernels()) >= 1
assert norm_grad(dx=0, dx_stride=0) == OK and norm_grad(dgamma=0, dbeta=0) == OK
''')


def test_clip_refuses():
    run(r'''
refuses(clip(count=-1), "count")
assert lib.rg_clip_grad_norm(c, None, i32(3), f32(1.0), p(address()), None) == INVALID
refuses(clip(max_norm=-1.0), "max_norm")
refuses(clip(max_norm=math.nan), "max_norm")
refuses(clip(norm=0), "norm")
refuses(clip(norm=0x7002), "norm")
refuses(clip(sizes=(5, -1)), "tensor 1")
refuses(clip(sizes=((1 << 40) - 5, 7)), "tensor 1")
refuses(clip(types=(0, 3)), "tensor 1: unknown type")
refuses(clip(ins=(0x8000, 0)), "tensor 1: null")
refuses(clip(outs=(0, 0x8000)), "tensor 0: null")
refuses(clip(ins=(0x8000, 0x8001), types=(F32, BF16)), "tensor 1: pointer")
assert clip(sizes=()) == OK and clip(sizes=(0, 0), ins=(0, 0), outs=(0, 0)) == OK and clip(max_norm=math.inf) == OK
''')


@pytest.mark.parametrize("call,small,large", [("matmul_grad", "n=3000", "n=2_000_000, out_dim=900, dy_stride=900"), ("norm_grad", "n=1000", "n=2_000_000, dim=900, x_stride=900, dy_stride=900, dx_stride=900"),
                                              ("clip", "sizes=(9, 8)", "sizes=(9,) * 500")])
def test_scratch_outlives_graphs_and_is_refused_inside_them(call, small, large):
    """Growing keeps what a graph may hold; inside a recording a call that wants more is refused before it launches anything."""
    run(rf'''
S = 0x51
assert {call}({small}, stream=S) == OK
rt.forget()
rt.begin_capture(p(S))
assert {call}({small}, stream=S) == OK and not log("malloc"), message()
recorded = kernels()
status = {call}({large}, stream=S)
assert status == STATE and "records a graph" in message() and not kernels(), (status, message())
rt.end_capture()
assert {call}({large}, stream=S) == OK
lines = log()
assert any(x.startswith("malloc") for x in lines) and not any(x.startswith("free") or x.startswith("sync") for x in lines), lines
rt.begin_capture(p(S))
assert {call}({large}, stream=S) == OK and not log("malloc")
rt.end_capture()
held = rt.memory_held()
lib.rg_destroy(c)
assert rt.memory_held() == 0 and held > 0
''')


def test_calls_without_memory_fail_and_work_again():
    run(r'''
held = rt.memory_held()
rt.limit_memory(held)
for call in (lambda: matmul_grad(n=2_000_000, out_dim=900, dy_stride=900), norm_grad, lambda: clip(sizes=(100_000,))):
    assert call() == OOM and not kernels(), message()
rt.limit_memory((1 << 64) - 1)
for call in (lambda: matmul_grad(n=2_000_000, out_dim=900, dy_stride=900), norm_grad, lambda: clip(sizes=(100_000,))):
    assert call() == OK
''')


def test_launches_stay_within_the_device_limits():
    """Largest sizes: less than 2^32 threads to a launch, LDS within 64 KiB."""
    run(r'''
N = (1 << 31) - 1
assert quantize(n=N, dim=1, x_stride=1, packed_stride=5) == OK and quantize(n=N, dim=65536, x_stride=65536, packed_stride=8704) == OK
assert dequantize(n=N, dim=1, x_stride=1, packed_stride=5) == OK and dequantize(n=N, dim=65536, x_stride=65536, packed_stride=8704) == OK
assert matmul(n=N, dim=64) == OK and matmul(n=N, out_dim=65536, y_stride=65536) == OK and matmul(n=1, out_dim=65536, y_stride=65536) == OK
assert matmul_grad(n=N) == OK and matmul_grad(n=N, out_dim=65536, dy_stride=65536, dim=65536, rows_stride=8704, grad_stride=65536) == OK
for dim in (1, 16, 1024, 1025, 2048, 65536):
    assert norm(n=N, dim=dim, x_stride=dim, y_stride=dim) == OK
    assert norm_grad(n=N, dim=dim, x_stride=dim, dy_stride=dim, dx_stride=dim) == OK
assert clip(sizes=((1 << 39), 5)) == OK
for line in log("launch"):
    at = line.rsplit(" ", 5)
    x, y, block, lds = (int(v) for v in at[1:5])
    assert 1 <= x < 1 << 31 and 1 <= y <= 65535 and x * block < 1 << 32 and lds <= 65536, line
''')


def test_binding_counts_the_words_of_a_row_as_the_library_does():
    from paper_2505_10806_amd import binding as B
    for dim in list(range(1, 700)) + [1024, 65535, 65536]:
        assert B.mx4_row_words(dim) == B._lib.rg_mx4_row_words(dim)
    for dim in (0, -3, 65537):
        assert B._lib.rg_mx4_row_words(dim) == 0
        with pytest.raises(ValueError):
            B.mx4_row_words(dim)
