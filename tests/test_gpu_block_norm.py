"""moespec_block_norm against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from paper_2602_16052_amd import binding as mb

from attention_common import CODE, HALF_STEP, TORCH, f64

pytestmark = pytest.mark.gpu


def layer(d, dtype):
    return mb.LayerDesc(d, 1, 1, d, CODE[dtype], False)


def check(dtype, M, d, kind, sigmoid=False, post=True, weights=True, residual=True, scale=0.7, eps=1e-6, seed=0, magnitude=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    dt = TORCH[dtype]
    y, res = (rand(M, d) * magnitude).to(dt), (3 * rand(M, d)).to(dt) if residual else None
    gate = {mb.BLOCK_GATE_NONE: None, mb.BLOCK_GATE_CHANNEL: rand(d), mb.BLOCK_GATE_TOKEN: rand(M),
            mb.BLOCK_GATE_ELEMENT: rand(M, d)}[kind]
    gate = None if gate is None else gate.to(dt)
    w_post, w_pre = ((1 + 0.2 * rand(d)).to(dt), (1 + 0.2 * rand(d)).to(dt)) if weights else (None, None)
    w_post = w_post if post else None
    r, x = mb.moespec_block_norm(layer(d, dtype), y, res, post_norm=post, w_post=w_post, gate=gate, gate_kind=kind,
                                 gate_sigmoid=sigmoid, scale=scale, w_pre=w_pre, eps=eps)
    g64 = None if gate is None else f64(gate)[:, None] if kind == mb.BLOCK_GATE_TOKEN else f64(gate)
    wr, wx, z = A.block_norm(f64(y), None if res is None else f64(res), post, None if w_post is None else f64(w_post), g64, sigmoid,
                             float(np.float32(scale)), None if w_pre is None else f64(w_pre), float(np.float32(eps)))
    # z: mean square of up to 32 squares a thread and 8 sums of pairs (half of it through the root), some ten roundings, the
    # hardware exponential of the sigmoid (2^-21); r adds one
    f32 = (20 + 20) * 2.0 ** -24 + 2.0 ** -21
    tol_r = HALF_STEP[dtype] * np.abs(wr) * (1 + 2.0 ** -6) + f32 * (z + np.abs(wr))
    assert np.all(np.abs(f64(r) - wr) <= tol_r), np.max(np.abs(f64(r) - wr) / tol_r)
    # x: an element of r is off by f32 (z + |r|), its norm by f32 relative
    norm = np.abs(wx) / np.maximum(np.abs(wr), 1e-300)
    tol_x = HALF_STEP[dtype] * np.abs(wx) * (1 + 2.0 ** -6) + f32 * norm * (z + np.abs(wr)) + 3 * f32 * np.abs(wx)
    assert np.all(np.abs(f64(x) - wx) <= tol_x), np.max(np.abs(f64(x) - wx) / tol_x)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", [mb.BLOCK_GATE_NONE, mb.BLOCK_GATE_CHANNEL, mb.BLOCK_GATE_TOKEN, mb.BLOCK_GATE_ELEMENT])
@pytest.mark.parametrize("d", [32, 96, 1024, 2016, 2080, 4096, 8192])
def test_gates_and_sizes(dtype, kind, d):
    check(dtype, 5, d, kind, seed=d + kind)
    check(dtype, 1, d, kind, sigmoid=True, seed=d)


@pytest.mark.parametrize("d", [4, 12, 1028, 4100])
def test_f32_rows_of_four(d):
    check("f32", 3, d, mb.BLOCK_GATE_CHANNEL, seed=d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_options(dtype):
    check(dtype, 4, 256, mb.BLOCK_GATE_NONE, post=False)
    check(dtype, 4, 256, mb.BLOCK_GATE_ELEMENT, post=False, residual=False)
    check(dtype, 4, 256, mb.BLOCK_GATE_NONE, weights=False, scale=-2.5)
    check(dtype, 4, 256, mb.BLOCK_GATE_NONE, weights=False, eps=0.0)
    check(dtype, 4, 256, mb.BLOCK_GATE_NONE, magnitude=1e-4, eps=1e-5)
    check(dtype, 700, 512, mb.BLOCK_GATE_TOKEN, sigmoid=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_alone_and_in_place(dtype):
    d, dt = 512, TORCH[dtype]
    y, res, gate = (torch.randn((9, d), device="cuda").to(dt) for _ in range(3))
    kw = dict(post_norm=True, gate_kind=mb.BLOCK_GATE_ELEMENT, scale=0.5, eps=1e-6)
    r, x = mb.moespec_block_norm(layer(d, dtype), y, res, gate=gate, **kw)
    only = torch.empty_like(y)
    mb.BlockNormCall(layer(d, dtype), y, res, only, None, gate=gate, **kw)()
    assert torch.equal(only, r)
    mb.BlockNormCall(layer(d, dtype), y, res, None, only, gate=gate, **kw)()
    assert torch.equal(only, x)
    for r_at, x_at in ((0, 1), (1, 0), (2, 0), (1, 2)):
        b = [y.clone(), res.clone(), gate.clone()]
        mb.BlockNormCall(layer(d, dtype), b[0], b[1], b[r_at], b[x_at], gate=b[2], **kw)()
        assert torch.equal(b[r_at], r) and torch.equal(b[x_at], x)


def test_non_finite_rows_stay_in_their_rows_and_zero_rows_with_eps():
    y, res = torch.randn((4, 64), device="cuda").bfloat16(), torch.randn((4, 64), device="cuda").bfloat16()
    y[1, 3], y[2] = float("nan"), 0
    res[2] = 0
    r, x = mb.moespec_block_norm(layer(64, "bf16"), y, res, post_norm=True, eps=1e-6)
    assert torch.isnan(r[1]).all() and torch.isnan(x[1]).all()
    assert torch.all(r[2] == 0) and torch.all(x[2] == 0)
    assert torch.isfinite(r[[0, 2, 3]]).all() and torch.isfinite(x[[0, 2, 3]]).all()


def test_captured_call_and_other_stream():
    d = layer(2048, "bf16")
    y, res = torch.randn((63, 2048), device="cuda").bfloat16(), torch.randn((63, 2048), device="cuda").bfloat16()
    r, x = torch.empty_like(y), torch.empty_like(y)
    call = mb.BlockNormCall(d, y, res, r, x, post_norm=True, eps=1e-6)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        y.mul_(0.5).add_(0.25)
        want = mb.moespec_block_norm(d, y, res, post_norm=True, eps=1e-6)
        r.zero_(), x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(r, want[0]) and torch.equal(x, want[1])
