"""The calls of learned vectors over the recording runtime, without a GPU: what they refuse, and what becomes of their scratch."""
import pytest

import host_calls

_CALLS = r'''
import math
INVALID, STATE = 1, 5
F32, BF16, F16 = 0, 1, 2
f32 = ctypes.c_float
c = context()
def message(): return lib.rg_last_error(c).decode()
def a(v): return p(address() if v is None else v)
def lookup(table=None, type=F32, stride=100, rows=50, ids=None, n=10, n_dev=0, dim=100, scale=1.0, y=None, y_type=F32, y_stride=100, stream=0):
    return lib.rg_embedding(c, a(table), i32(type), i64(stride), i64(rows), a(ids), i64(n), p(n_dev), i32(dim), f32(scale), a(y), i32(y_type), i64(y_stride), p(stream))
def grad(dy=None, type=F32, stride=100, ids=None, n=10, n_dev=0, dim=100, rows=50, scale=1.0, add=0, grad=None, grad_type=F32, grad_stride=100, stream=0):
    return lib.rg_embedding_grad(c, a(dy), i32(type), i64(stride), a(ids), i64(n), p(n_dev), i32(dim), i64(rows), f32(scale), i32(add), a(grad), i32(grad_type),
                                 i64(grad_stride), p(stream))
def grad_rows(dy=None, type=F32, stride=100, ids=None, n=10, n_dev=0, dim=100, rows=50, scale=1.0, grad=None, grad_stride=100, touched=None, met=None, stream=0):
    return lib.rg_embedding_grad_rows(c, a(dy), i32(type), i64(stride), a(ids), i64(n), p(n_dev), i32(dim), i64(rows), f32(scale), a(grad), i64(grad_stride),
                                      a(touched), a(met), p(stream))
def loss(x=None, type=F32, stride=100, n=10, n_dev=0, dim=100, weight=None, weight_stride=100, classes=30, labels=None, loss=None, lse=None, stream=0):
    return lib.rg_cross_entropy(c, a(x), i32(type), i64(stride), i64(n), p(n_dev), i32(dim), a(weight), i64(weight_stride), i32(classes), a(labels), a(loss),
                                a(lse), p(stream))
def loss_grad(x=None, type=F32, stride=100, n=10, n_dev=0, dim=100, weight=None, weight_stride=100, classes=30, labels=None, lse=None, dloss=0, scale=1.0,
              dx=None, dx_stride=100, dweight=None, dweight_stride=100, stream=0):
    return lib.rg_cross_entropy_grad(c, a(x), i32(type), i64(stride), i64(n), p(n_dev), i32(dim), a(weight), i64(weight_stride), i32(classes), a(labels),
                                     a(lse), p(dloss), f32(scale), a(dx), i64(dx_stride), a(dweight), i64(dweight_stride), p(stream))
def refuses(status, text):
    assert status == INVALID and text in message(), (status, message())
    assert not kernels()
'''


def run(program):
    return host_calls.run(_CALLS + program)


def test_lookup_and_its_gradients_refuse():
    run(r'''
for call in (lookup, grad, grad_rows):
    refuses(call(n=-1), "out of range")
    refuses(call(n=1 << 31), "out of range")
    refuses(call(rows=-1), "out of range")
    refuses(call(rows=1 << 31), "out of range")
    refuses(call(dim=0), "dim")
    refuses(call(dim=65537, stride=70000), "dim")
    refuses(call(type=3), "type")
    refuses(call(stride=99), "stride")
    refuses(call(scale=math.nan), "scale")
    refuses(call(ids=0), "null")
    refuses(call(ids=0x7002), "aligned")
refuses(lookup(rows=0), "out of range")
refuses(lookup(table=0), "null")
refuses(lookup(y=0), "null")
refuses(lookup(y_type=-1), "type")
refuses(lookup(y_stride=99), "stride")
refuses(lookup(table=0x7002), "aligned")
refuses(lookup(y=0x7001, y_type=BF16), "aligned")
for call in (grad, grad_rows):
    refuses(call(dy=0), "null")
    refuses(call(grad=0), "null")
    refuses(call(grad=0x7002), "aligned")
    refuses(call(grad_stride=99), "stride")
    refuses(call(dy=0x7001, type=F16), "aligned")
refuses(grad(grad_type=7), "type")
refuses(lookup(table=0x8000, y=0x8000), "input")
refuses(grad(dy=0x8000, grad=0x8000), "input")
refuses(grad_rows(dy=0x8000, grad=0x8000), "input")
refuses(grad_rows(ids=0x8000, touched=0x8000), "input")
refuses(grad_rows(touched=0x8000, met=0x8000), "output")
refuses(grad_rows(touched=0), "null")
refuses(grad_rows(met=0), "null")
refuses(grad_rows(met=0x7001), "aligned")
refuses(grad_rows(touched=0x7001), "aligned")
assert lookup(n=0, table=0, ids=0, y=0) == OK and grad(rows=0, grad=0) == OK and grad(n=0, dy=0, ids=0, add=1) == OK and not kernels()
assert grad(n=0, dy=0, ids=0) == OK and len(kernels()) == 1                      # zeros
assert grad_rows(n=0, dy=0, ids=0, grad=0, touched=0) == OK and len(kernels()) == 1  # none met
assert grad_rows(rows=0, grad=0, touched=0) == OK and len(kernels()) == 1
assert lookup(table=0x7002, type=F16, y=0x7006, y_type=BF16) == OK
''')


def test_loss_and_its_gradient_refuse():
    run(r'''
for call in (loss, loss_grad):
    refuses(call(n=-1), "out of range")
    refuses(call(n=1 << 31), "out of range")
    refuses(call(dim=0), "dim")
    refuses(call(dim=65537, stride=70000, weight_stride=70000), "dim")
    refuses(call(classes=0), "classes")
    refuses(call(classes=-5), "classes")
    refuses(call(type=3), "type")
    refuses(call(stride=99), "stride")
    refuses(call(weight_stride=99), "stride")
    refuses(call(x=0), "null")
    refuses(call(weight=0), "null")
    refuses(call(labels=0), "null")
    refuses(call(x=0x7002), "aligned")
    refuses(call(weight=0x7001, type=BF16), "aligned")
    refuses(call(labels=0x7002), "aligned")
    refuses(call(lse=0x7002), "aligned")
refuses(loss(loss=0x7002), "aligned")
refuses(loss_grad(lse=0), "null")
refuses(loss_grad(dloss=0x7002), "aligned")
refuses(loss_grad(dx_stride=99), "stride")
refuses(loss_grad(dweight_stride=99), "stride")
refuses(loss_grad(dx=0x7002), "aligned")
refuses(loss_grad(dweight=0x7001, type=F16), "aligned")
refuses(loss_grad(scale=math.nan), "scale")
refuses(loss(classes=(1 << 30) + 1), "classes")
refuses(loss_grad(classes=(1 << 30) + 1), "classes")
refuses(loss_grad(x=0x8000, dx=0x8000), "input")
refuses(loss_grad(weight=0x8000, dweight=0x8000), "input")
refuses(loss_grad(dx=0x8000, dweight=0x8000), "output")
assert loss(n=0, x=0, weight=0, labels=0) == OK and loss(loss=0, lse=0) == OK and loss_grad(dx=0, dweight=0) == OK and not kernels()
assert loss_grad(n=0, x=0, weight=0, labels=0, lse=0, dweight=0) == OK and not kernels()
assert loss_grad(n=0, x=0, weight=0, labels=0, lse=0) == OK and len(kernels()) == 1       # zeros
assert loss(x=0x7002, weight=0x7006, type=F16) == OK and loss_grad(dx=0, dx_stride=0) == OK and loss_grad(dweight=0, dweight_stride=0) == OK
''')


@pytest.mark.parametrize("call,small,large", [("grad", "n=3000", "n=2_000_000"), ("grad_rows", "n=3000", "n=2_000_000, rows=1 << 30"),
                                              ("loss", "n=300", "n=20_000, classes=100_000"), ("loss_grad", "n=300", "n=20_000, classes=100_000")])
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
rt.limit_memory(rt.memory_held())
for call in (grad, grad_rows, lambda: loss(classes=300), loss_grad):
    assert call() == OOM and not kernels(), message()
rt.limit_memory((1 << 64) - 1)
for call in (grad, grad_rows, lambda: loss(classes=300), loss_grad):
    assert call() == OK
''')


def test_launches_stay_within_the_device_limits():
    """Largest sizes: less than 2^32 threads to a launch, LDS that is asked for at a launch within 64 KiB."""
    run(r'''
N = (1 << 31) - 1
for dim in (1, 100, 65536):
    for t in (F32, BF16):
        assert lookup(n=N, rows=N, dim=dim, stride=dim, y_stride=dim, type=t) == OK
        assert grad(n=N, rows=N, dim=dim, stride=dim, grad_stride=dim, type=t) == OK and grad_rows(n=N, rows=N, dim=dim, stride=dim, grad_stride=dim, type=t) == OK
        assert grad(n=1, rows=N, dim=dim, stride=dim, grad_stride=dim, type=t) == OK and grad(n=0, rows=N, dim=dim, grad_stride=dim, stride=dim) == OK
for dim, most in ((1, 1 << 30), (100, 1 << 27), (300, 1 << 25), (65536, 100_000)):
    for t in (F32, BF16):
        for n, classes in ((most, 1), (1, most), (1 << 20, 1 << 20) if dim < 65536 else (3000, 3000), (1, 1)):
            assert loss(n=n, classes=classes, dim=dim, stride=dim, weight_stride=dim, type=t) == OK and loss(n=30, classes=most, dim=dim, stride=dim, weight_stride=dim, type=t) == OK
            assert loss(n=most, classes=50, dim=dim, stride=dim, weight_stride=dim, type=t) == OK
            assert loss_grad(n=most, classes=50, dim=dim, stride=dim, weight_stride=dim, dx_stride=dim, dweight_stride=dim, type=t) == OK
            assert loss_grad(n=n, classes=classes, dim=dim, stride=dim, weight_stride=dim, dx_stride=dim, dweight_stride=dim, type=t) == OK
for line in log("launch"):
    at = line.rsplit(" ", 5)
    x, y, block, lds = (int(v) for v in at[1:5])
    assert 1 <= x < 1 << 31 and 1 <= y <= 65535 and x * block < 1 << 32 and lds <= 65536, line
''')


def test_scratch_of_long_walks_is_bounded():
    """Gradients of f32 that are cut into walks of at most 4096 rows: parts of a gigabyte, twice that where their number is rounded up, and the owned rows' 128 MB."""
    run(r'''
for dim in (1, 16, 100, 300, 4000, 65536):
    most = min((1 << 31) - 1, (1 << 38) // dim)
    for n, classes in ((most, 65), (most, 4097), (most, 70_000), (40, min(1 << 30, most)), (33_000, min(1 << 30, most)), (1 << 20, min(1 << 30, most)), (5000, 5000), (70_000, 70_000)):
        held = rt.memory_held()
        assert loss_grad(n=n, classes=classes, dim=dim, stride=dim, weight_stride=dim, dx_stride=dim, dweight_stride=dim, type=F32) == OK, message()
        assert rt.memory_held() - held <= (2 << 30) + (160 << 20), (n, classes, dim, rt.memory_held() - held)
        rt.forget()
        lib.rg_destroy(c)
        c = context()
''')
