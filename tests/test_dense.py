"""Uncompressed layers on the host side: plans, refusals, cache layout and workspace sizes (no
GPU: nothing here launches a kernel), and the float64 reference that the GPU tests compare with."""
import ctypes as C
import math

import pytest
import torch

import _dense_ref as R
from paper_2606_08382_amd import starkv as S

FAKE = 1 << 40            # never dereferenced: every call below fails validation first


def status(fn, *args, **kw):
    with pytest.raises(S.StarkvError) as e:
        fn(*args, **kw)
    assert S.starkv_last_error()
    return e.value.status


def rope_cfg(**kw):
    base = dict(head_dim=128, theta=1e4)
    base.update(kw)
    return S.make_rope_config(**base)


@pytest.mark.parametrize("kw,st", [
    (dict(head_dim=0), 1), (dict(head_dim=63), 1), (dict(head_dim=514), 2),
    (dict(rotary_dim=0), 1), (dict(rotary_dim=31), 1), (dict(rotary_dim=130), 1),
    (dict(layout=2), 1), (dict(scaling=5), 1), (dict(scaling=-1), 1), (dict(dtype=3), 1),
    (dict(theta=1.0), 1), (dict(theta=math.inf), 1), (dict(theta=math.nan), 1),
    (dict(scaling=S.ROPE_LINEAR, factor=0.5), 1), (dict(scaling=S.ROPE_NTK, factor=math.nan), 1),
    (dict(scaling=S.ROPE_NTK, factor=2.0, rotary_dim=2), 1), (dict(gain=-1.0), 1),
    (dict(scaling=S.ROPE_BANDS, factor=2.0), 1),
    (dict(scaling=S.ROPE_YARN, factor=2.0, original_ctx=64, turns_low=3.0, turns_high=2.0), 1),
])
def test_rope_plan_refuses(kw, st):
    assert status(S.starkv_rope_plan_create, rope_cfg(**kw)) == st


def test_rope_refuses():
    plan = S.starkv_rope_plan_create(rope_cfg())
    st = S.starkv_strides

    def call(x=FAKE, xs=None, out=FAKE + 512, os_=None, pos=FAKE, b=2, n=3, h=4):
        return status(S.starkv_rope, plan, x, xs, out, os_, pos, b, n, h)
    assert call(x=None) == call(out=None) == call(pos=None) == 1
    assert call(b=0) == call(n=0) == call(h=0) == call(b=-1) == 1
    assert call(x=FAKE + 1) == call(out=FAKE + 1) == call(pos=FAKE + 2) == 5
    assert call(os_=st(128 * 12, 128 * 4, 64)) == 1           # heads of out overlap
    assert call(os_=st(128 * 12, 0, 128)) == 1
    assert call(out=FAKE, os_=st(128 * 12, 128 * 4, 256)) == 1   # in place, other strides


def dense_cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, capacity=1000, n_blocks=80,
                block_table=FAKE)
    base.update(kw)
    return S.make_dense_config(**base)


@pytest.mark.parametrize("kw,st", [
    (dict(batch=0), 1), (dict(n_q_heads=0), 1), (dict(n_kv_heads=0), 1), (dict(n_q_heads=7), 1),
    (dict(capacity=0), 1), (dict(code=2), 1), (dict(code=-1), 1), (dict(dtype=S.DT_F32), 1),
    (dict(block_tokens=8), 1), (dict(block_tokens=48), 1), (dict(block_tokens=256), 1),
    (dict(n_blocks=0), 1), (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=math.inf), 1),
    (dict(block_table=None), 1), (dict(block_table=FAKE + 2), 5), (dict(batch=32768), 2),
    (dict(n_q_heads=34, n_kv_heads=17), 2), (dict(n_q_heads=66), 2), (dict(head_dim=96), 2),
    (dict(capacity=524289), 2), (dict(n_blocks=1 << 30), 2),
])
def test_dense_plan_refuses(kw, st):
    assert status(S.starkv_dense_plan_create, dense_cfg(**kw)) == st


def test_null_configs_and_plans():
    L = S.lib()
    h = C.c_void_p()
    for create in (L.starkv_rope_plan_create, L.starkv_dense_plan_create):
        assert create(None, C.byref(h)) == 1
        assert not h.value
    L.starkv_rope_plan_destroy(None)
    L.starkv_dense_plan_destroy(None)
    assert L.starkv_dense_cache_bytes(None) == 0
    assert L.starkv_dense_workspace_bytes(None, 1, 1, 0) == 0
    assert L.starkv_dense_attn(None, FAKE, FAKE, None, 1, None, FAKE, 1, FAKE, None, None, FAKE,
                               0, None) == 1
    assert L.starkv_dense_evict(None, FAKE, FAKE, 1, 0, 0, None, None, None, None) == 1


def test_dense_entry_points_refuse():
    plan = S.starkv_dense_plan_create(dense_cfg())
    st = S.starkv_strides

    def append(cache=FAKE, k=FAKE, ks=None, v=FAKE, vs=None, pos=FAKE, n=1, n_dev=None):
        return status(S.starkv_dense_append, plan, cache, k, ks, v, vs, pos, n, n_dev)
    assert append(cache=None) == append(k=None) == append(v=None) == append(pos=None) == 1
    assert append(n=0) == append(n=-3) == 1
    assert append(cache=FAKE + 128) == append(k=FAKE + 1) == append(v=FAKE + 1) == 5
    assert append(pos=FAKE + 2) == append(n_dev=FAKE + 1) == 5

    def read(cache=FAKE, ctx=FAKE, start=FAKE, n=1, k=FAKE, ks=None, v=FAKE, vs=None, dt=0):
        return status(S.starkv_dense_read, plan, cache, ctx, start, n, k, ks, v, vs, dt)
    assert read(ctx=None) == read(start=None) == read(n=0) == read(dt=3) == 1
    assert read(k=None, v=None) == 1
    assert read(k=FAKE + 2, dt=S.DT_F32) == read(v=FAKE + 1) == read(cache=FAKE + 8) == 5
    assert read(n=2, ks=st(1000, 100, 128)) == 1

    need = S.starkv_dense_workspace_bytes(plan, 2, 1000, True)

    def attn(cache=FAKE, q=FAKE, qs=None, n=2, q_len=None, ctx=FAKE, most=1000, out=FAKE, os_=None,
             w=FAKE, ws=FAKE, nbytes=need):
        return status(S.starkv_dense_attn, plan, cache, q, qs, n, q_len, ctx, most, out, os_, w,
                      ws, nbytes)
    assert attn(cache=None) == attn(q=None) == attn(ctx=None) == attn(out=None) == 1
    assert attn(n=0) == attn(most=0) == 1
    assert attn(most=1001) == 3
    assert attn(n=17) == 2                                # weights: 17 * 4 rows > 64
    assert attn(n=1 << 20, w=None) == 2
    assert attn(ws=None) == attn(nbytes=need - 1) == 4
    assert attn(ws=FAKE + 64) == attn(q=FAKE + 1) == attn(out=FAKE + 1) == 5
    assert attn(ctx=FAKE + 1) == attn(q_len=FAKE + 2) == attn(w=FAKE + 2) == 5
    assert attn(os_=st(2048, 1024, 64)) == 1

    def evict(w=FAKE, ctx=FAKE, keep=4, sink=1, recent=1, t=None, wo=None, co=None):
        return status(S.starkv_dense_evict, plan, w, ctx, keep, sink, recent, t, wo, co)
    assert evict(w=None) == evict(ctx=None) == 1
    assert evict(keep=0, sink=0, recent=0) == evict(sink=-1) == evict(recent=-1) == 1
    assert evict(sink=3, recent=2) == evict(sink=2 ** 31 - 1, recent=2 ** 31 - 1) == 1
    assert evict(w=FAKE + 1) == evict(ctx=FAKE + 1) == evict(t=FAKE + 1) == 5
    assert evict(wo=FAKE + 2) == evict(co=FAKE + 2) == 5


@pytest.mark.parametrize("d,T,cap,blocks", [(128, 64, 1000, 80), (64, 16, 17, 9), (128, 128, 1, 1)])
def test_dense_layout(d, T, cap, blocks):
    plan = S.starkv_dense_plan_create(dense_cfg(head_dim=d, block_tokens=T, capacity=cap,
                                                n_blocks=blocks))
    L = S.starkv_dense_cache_layout(plan)

    def up(x):
        return -(-x // 256) * 256
    assert L.blocks_per_head == -(-cap // T)
    assert L.block_bytes == 2 * T * d and L.tail_bytes == 2 * (2 * T) * d * 2
    assert L.code_offset == 0 and L.scale_offset == up(blocks * 2 * T * d)
    assert L.tail_offset == L.scale_offset + up(8 * blocks)
    assert L.total_bytes == L.tail_offset + up(2 * 2 * L.tail_bytes)
    assert S.starkv_dense_cache_bytes(plan) == L.total_bytes


@pytest.mark.parametrize("batch", [2, 40, 300])
@pytest.mark.parametrize("heads", [(8, 8), (8, 1), (32, 8), (64, 1), (6, 2)])
def test_workspace_serves_fewer_tokens_and_shorter_contexts(heads, batch):
    plan = S.starkv_dense_plan_create(dense_cfg(n_q_heads=heads[0], n_kv_heads=heads[1],
                                                capacity=5000, batch=batch))
    sizes = {(n, ctx, w): S.starkv_dense_workspace_bytes(plan, n, ctx, w)
             for n in (1, 2, 3, 5, 8, 16, 17, 33, 64, 200, 1000) for ctx in (1, 16, 17, 777, 5000)
             for w in (False, True)}
    for (n, ctx, w), size in sizes.items():
        assert size > 0
        for (n2, ctx2, w2), less in sizes.items():
            if n2 <= n and ctx2 <= ctx and w2 <= w:
                assert less <= size, (n, ctx, w, n2, ctx2, w2)
    assert S.starkv_dense_workspace_bytes(plan, 0, 10, False) == 0
    assert S.starkv_dense_workspace_bytes(plan, 1, 0, False) == 0


def test_layers_refuse_host_memory():
    from paper_2606_08382_amd.device import DenseLayer, Rope
    table = torch.zeros((1, 1, 1), dtype=torch.int32)
    with pytest.raises(ValueError):
        DenseLayer(1, 1, 1, 64, 16, block_tokens=16, block_table=table)
    rope = Rope(64, 1e4)
    with pytest.raises(ValueError):
        rope(torch.zeros(1, 2, 64), torch.zeros(1, dtype=torch.int32))


# ------------------------------------------------------------ the reference, by its properties

@pytest.mark.parametrize("code", [0, 1])
def test_reference_quantizer(code):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 16, 64, generator=g, dtype=torch.float64).bfloat16()
    v, s = R.quantize(x, code)
    y = v * s.double()[:, None, None]
    err = (y - x.double()).abs()
    if code == 0:                             # half a step of the scale
        assert (err <= s.double()[:, None, None] / 2 * (1 + 2.0 ** -20)).all()
    else:                                     # half a step relative, or half the smallest step
        lim = torch.maximum(x.double().abs() * 2.0 ** -4, s.double()[:, None, None] * 2.0 ** -10)
        assert (err <= lim * (1 + 2.0 ** -20)).all()
        # the fp32 quotient rounds to the same code unless fp32 moved it onto a border (x and the
        # maximum have few bits, so x/s often lies 2^-24 from one)
        q = (x.double() / s.double()[:, None, None]).float()
        off = q.to(torch.float8_e4m3fn).double() != v
        g = R.grid(code)
        assert torch.isin(q[off].double().abs(), (g[1:] + g[:-1]) / 2).all()
    assert torch.isnan(R.quantize(torch.full((1, 16, 64), math.inf), code)[1]).all()


def test_reference_rope_is_a_rotation():
    x = torch.randn(3, 2, 8, dtype=torch.float64)
    pos = torch.tensor([0, 5, 100000])
    f = R.rope_turns(6, 1e4, 0)
    for il in (False, True):
        y = R.rope(x, pos, f, il)
        assert torch.equal(y[0], x[0]) and torch.equal(y[..., 6:], x[..., 6:])
        assert torch.allclose(y.square().sum(-1), x.square().sum(-1))
        assert torch.allclose(R.rope(y, pos, f, il, inverse=True), x)


def test_reference_evict():
    t, w, n = R.evict([5., 1., 3., 2., 4., 9.], [10, 11, 12, 13, 14, 15], 5 * 16 + 3, 16, 3, 1, 1)
    assert (t, w, n) == ([10, 12, 14, 11, 13, 15], [5., 3., 4., 9., 0., 0.], 3 * 16 + 3)
    t, w, n = R.evict([1.0] * 4, [0, 1, 2, 3], 64, 16, 1, 0, 0)     # an even number leaves
    assert (t, w, n) == ([0, 1, 2, 3], [1.0, 1.0, 0.0, 0.0], 32)
