"""Refusals of the training-step calls, all on the host (no GPU needed): fake
pointers are never dereferenced, CPU tensors never passed on."""

import ctypes

import pytest
import torch

gift = pytest.importorskip("paper_2607_07494_amd.gift")
LIB = gift.LIB
FAKE = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1001)
E, S = gift.EINVAL, gift.ESHAPE
NAN, INF = float("nan"), float("inf")


@pytest.fixture
def ctx():
    c = gift.Context(stream=0)   # creating a context makes no HIP call
    yield c
    c.close()


def _err():
    return LIB.gift_last_error().decode()


LOOKUP = dict(table=FAKE, td=0, V=10, d=4, tokens=FAKE, it=0, T=3, scale=1.0, out=FAKE, od=0)


@pytest.mark.parametrize("change,status,word", [
    (dict(table=None), E, "NULL"), (dict(tokens=None), E, "NULL"), (dict(out=None), E, "NULL"),
    (dict(td=2), E, "dtypes"), (dict(od=-1), E, "dtypes"), (dict(it=2), E, "token_type"),
    (dict(scale=NAN), E, "scale"), (dict(scale=INF), E, "scale"),
    (dict(T=-1), S, "T must"), (dict(T=1 << 31), S, "T must"), (dict(V=0), S, "V must"), (dict(V=(1 << 31) - 1), S, "V must"),
    (dict(d=0), S, "d must"), (dict(d=(1 << 20) + 1), S, "d must"),
    (dict(table=ODD), E, "aligned"), (dict(out=ODD, od=1), E, "aligned"), (dict(tokens=ctypes.c_void_p(0x1004), it=1), E, "aligned"),
])
def test_embedding(ctx, change, status, word):
    assert LIB.gift_embedding(ctx.handle, *dict(LOOKUP, **change).values()) == status
    assert "gift_embedding" in _err() and word in _err()


def test_embedding_of_no_tokens_enqueues_nothing(ctx):
    assert LIB.gift_embedding(ctx.handle, *dict(LOOKUP, T=0, tokens=None, out=None).values()) == gift.OK
    assert LIB.gift_embedding(None, *LOOKUP.values()) == E


GRAD = dict(tokens=FAKE, it=0, dout=FAKE, dt=0, N=2, T=3, V=10, d=4, scale=1.0, acc=0, grads=FAKE, ws=None, bytes=0)


@pytest.mark.parametrize("change,status,word", [
    (dict(tokens=None), E, "NULL"), (dict(dout=None), E, "NULL"), (dict(grads=None), E, "NULL"),
    (dict(dt=2), E, "dtype"), (dict(it=-1), E, "token_type"), (dict(scale=-INF), E, "scale"),
    (dict(N=0), S, "N must"), (dict(N=65536), S, "N must"), (dict(T=-1), S, "T must"), (dict(T=1 << 30), S, "T must"),
    (dict(V=0), S, "V must"), (dict(d=0), S, "d must"), (dict(grads=ctypes.c_void_p(0x1002)), E, "aligned"),
    (dict(dout=ODD, dt=1), E, "aligned"), (dict(N=65535, V=1 << 30), S, "more work"),
])
def test_embedding_grad(ctx, change, status, word):
    assert LIB.gift_embedding_grad(ctx.handle, *dict(GRAD, **change).values()) == status
    assert "gift_embedding_grad" in _err() and word in _err()


def test_embedding_grad_scratch_sizes(ctx):
    assert LIB.gift_embedding_grad(None, *GRAD.values()) == E
    assert LIB.gift_embedding_grad(ctx.handle, *dict(GRAD, T=0, acc=1, tokens=None, dout=None).values()) == gift.OK
    f = gift.embedding_grad_scratch
    assert f(0, 8, 8, 8) == f(1, 0, 8, 8) == f(1, 8, 0, 8) == f(1, 8, 8, 0) == f(2, 1 << 30, 8, 8) == 0
    assert f(2, 100, 8, 8) >= 2 * 100 * 16


NORM = dict(count=2, grads=(ctypes.c_void_p * 2)(0x1000, 0x2000), numel=(ctypes.c_int64 * 2)(4, 5), dt=0, max_norm=1.0,
            out=FAKE, ws=None, bytes=0)


@pytest.mark.parametrize("change,status,word", [
    (dict(grads=None), E, "NULL"), (dict(numel=None), E, "NULL"), (dict(out=None), E, "NULL"), (dict(out=ODD), E, "aligned"),
    (dict(dt=3), E, "dtype"), (dict(max_norm=0.0), E, "max_norm"), (dict(max_norm=NAN), E, "max_norm"),
    (dict(count=-1), S, "count"), (dict(numel=(ctypes.c_int64 * 2)(4, -1)), S, "element counts"),
    (dict(numel=(ctypes.c_int64 * 2)(4, (1 << 33) + 1)), S, "element counts"),
    (dict(grads=(ctypes.c_void_p * 2)(0x1000, None)), E, "NULL"), (dict(grads=(ctypes.c_void_p * 2)(0x1000, 0x2002)), E, "aligned"),
])
def test_grad_norm(ctx, change, status, word):
    assert LIB.gift_grad_norm(ctx.handle, *dict(NORM, **change).values()) == status
    assert "gift_grad_norm" in _err() and word in _err()


def _step(ctx, tensor=None, count=1, null=False, **options):
    t = dict(param=0x1000, grad=0x2000, m=0x3000, v=0x4000, m_scales=0x5000, v_scales=0x6000, copy=0x7000, numel=5,
             weight_decay=0.1)
    t.update(tensor or {})
    o = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1, seed=0, grad_dtype=0, moments=0)
    o.update(options)
    tensors = (gift._AdamWTensor * 1)(gift._AdamWTensor(**t))
    return LIB.gift_adamw_step(ctx.handle if ctx else None, count, None if null else tensors,
                               ctypes.byref(gift._AdamWOptions(**o)))


@pytest.mark.parametrize("kw,status,word", [
    (dict(count=-1), S, "count"), (dict(null=True), E, "NULL"), (dict(grad_dtype=2), E, "grad_dtype"), (dict(moments=2), E, "moments"),
    (dict(lr=-1.0), E, "lr"), (dict(lr=NAN), E, "lr"), (dict(lr=INF), E, "lr"),
    (dict(beta1=1.0), E, "betas"), (dict(beta2=-0.1), E, "betas"), (dict(beta2=NAN), E, "betas"),
    (dict(eps=0.0), E, "eps"), (dict(eps=1e-60), E, "eps"), (dict(eps=1e60), E, "eps"), (dict(step=0), E, "step"),
    (dict(lr_dev=0x1002), E, "scalar"), (dict(step_dev=0x1004), E, "scalar"), (dict(grad_scale=0x1001), E, "scalar"),
    (dict(tensor=dict(param=None)), E, "NULL"), (dict(tensor=dict(grad=None)), E, "NULL"), (dict(tensor=dict(m=None)), E, "NULL"),
    (dict(tensor=dict(v_scales=None), moments=1), E, "NULL"),
    (dict(tensor=dict(numel=-1)), S, "element counts"), (dict(tensor=dict(numel=(1 << 33) + 1)), S, "element counts"), (dict(tensor=dict(weight_decay=-0.1)), E, "weight decays"),
    (dict(tensor=dict(weight_decay=INF)), E, "weight decays"), (dict(tensor=dict(param=0x1002)), E, "aligned"),
    (dict(tensor=dict(v=0x1002)), E, "aligned"), (dict(tensor=dict(copy=0x1001)), E, "aligned"),
    (dict(tensor=dict(m_scales=0x1002), moments=1), E, "aligned"), (dict(tensor=dict(grad=0x1001), grad_dtype=1), E, "aligned"),
])
def test_adamw_step(ctx, kw, status, word):
    assert _step(ctx, **kw) == status
    assert "gift_adamw_step" in _err() and word in _err()


def test_adamw_null_handles(ctx):
    assert _step(None) == E
    assert LIB.gift_adamw_step(ctx.handle, 0, None, None) == E


# ---------------------------------------------------------------- binding
def z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def test_binding_embedding(ctx):
    ids = z(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="2-dimensional"):
        gift.embedding(ctx, z(4), ids, z(3, 4))
    with pytest.raises(ValueError, match="must have shape"):
        gift.embedding(ctx, z(5, 4), ids, z(3, 5))
    with pytest.raises(TypeError, match="tokens"):
        gift.embedding(ctx, z(5, 4), z(3), z(3, 4))
    with pytest.raises(TypeError, match="table"):
        gift.embedding(ctx, z(5, 4, dtype=torch.float16), ids, z(3, 4))
    with pytest.raises(ValueError, match="GPU tensor"):
        gift.embedding(ctx, z(5, 4), ids, z(3, 4))


def test_binding_embedding_grad(ctx):
    ids = z(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="tokens must have shape"):
        gift.embedding_grad(ctx, z(1, 3, dtype=torch.int32), z(2, 3, 4), z(2, 5, 4))
    with pytest.raises(ValueError, match="dout must have shape"):
        gift.embedding_grad(ctx, ids, z(2, 3, 5), z(2, 5, 4))
    with pytest.raises(TypeError, match="grads"):
        gift.embedding_grad(ctx, ids, z(2, 3, 4), z(2, 5, 4, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="GPU tensor"):
        gift.embedding_grad(ctx, ids, z(2, 3, 4), z(2, 5, 4))


def test_binding_grad_norm(ctx):
    with pytest.raises(ValueError, match="out must have shape"):
        gift.grad_norm(ctx, [z(3)], z(1))
    with pytest.raises(TypeError, match="out must have dtype"):
        gift.grad_norm(ctx, [z(3)], z(2, dtype=torch.float64))
    with pytest.raises(ValueError, match="GPU tensor"):
        gift.grad_norm(ctx, [z(3)], z(2))


def test_binding_adamw(ctx):
    p = [z(3, 4)]
    with pytest.raises(ValueError, match="moments must be"):
        gift.AdamW(ctx, p, moments="int8")
    with pytest.raises(TypeError, match="float32"):
        gift.AdamW(ctx, [z(3, dtype=torch.bfloat16)])
    with pytest.raises(ValueError, match="one entry per parameter"):
        gift.AdamW(ctx, p, weight_decay=[0.1, 0.1])
    with pytest.raises(ValueError, match="a copy must have shape"):
        gift.AdamW(ctx, p, copies=[z(4, 3, dtype=torch.bfloat16)])
    with pytest.raises(TypeError, match="copies"):
        gift.AdamW(ctx, p, copies=[z(3, 4)])
    with pytest.raises(ValueError, match="state must hold"):
        gift.AdamW(ctx, p, state=dict(m=z(512)))
    with pytest.raises(ValueError, match="must have shape"):
        gift.AdamW(ctx, p, state=dict(m=z(12), v=z(12)))
    with pytest.raises(TypeError, match="must have dtype"):
        gift.AdamW(ctx, p, state=dict(m=z(512), v=z(512, dtype=torch.bfloat16)))
    with pytest.raises(ValueError, match="GPU tensor"):
        gift.AdamW(ctx, p)
    sizes = gift.AdamW.state_sizes([z(3, 4), z(513), z(0)], "e4m3")
    assert sizes["m"] == (512 + 1024, torch.uint8) and sizes["v_scales"] == (6, torch.float32)


def test_binding_adamw_step(ctx):
    opt = gift.AdamW(ctx, [])
    with pytest.raises(ValueError, match="one entry per parameter"):
        opt.step([z(3)], lr=0.1)
    with pytest.raises(TypeError, match="grad_scale must be a tensor"):
        opt.step([], lr=0.1, grad_scale=1.0)
    with pytest.raises(TypeError, match="lr must be one"):
        opt.step([], lr=z(2))
    with pytest.raises(TypeError, match="step must be one"):
        opt.step([], lr=0.1, step=z(1))
    opt.params, opt._shapes = [z(2, 2)], [torch.Size([2, 2])]
    with pytest.raises(ValueError, match="a gradient must have shape"):
        opt.step([z(4)], lr=0.1)
    with pytest.raises(gift.GiftError, match="lr must be"):
        opt.params, opt._shapes = [], []
        opt.step([], lr=-1.0)
    assert opt.steps == 0
