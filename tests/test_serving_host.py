"""The calls around a serving step without a GPU: argument checks and workspace sizes through the C ABI under sanitizers
(tests/host_checks_serving.c), the binding's checks of tensors, and the oracle against plain formulas."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
from oracle import serving_oracle as V
from paper_2602_16052_amd import binding as mb
from paper_2602_16052_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _clang():
    for cand in ("/opt/rocm/llvm/bin/clang", shutil.which("amdclang"), shutil.which("clang")):
        if cand and os.path.exists(cand):
            return cand
    return None


def test_argument_checks_are_clean_under_asan_and_ubsan(tmp_path):
    clang = _clang()
    if clang is None:
        pytest.skip("no clang to build the instrumented client with")
    lib = build.build_host_sanitizer_library(str(tmp_path))
    exe = str(tmp_path / "host_checks_serving")
    cc = subprocess.run([clang, "-std=c11", "-O1", "-g", "-Wall", "-Wextra", "-pedantic", "-Werror",
                         "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
                         "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host_checks_serving.c"),
                         lib, "-Wl,-rpath," + str(tmp_path), "-o", exe],
                        stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert cc.returncode == 0, cc.stdout
    env = dict(os.environ)
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=0:verify_asan_link_order=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1"
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=120)
    assert run.returncode == 0, run.stdout
    assert "host checks passed" in run.stdout
    assert "AddressSanitizer" not in run.stdout and "runtime error" not in run.stdout, run.stdout


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mb.LIB_PATH):
        build.build_library()
    return mb.load_library()


def test_binding_refuses_tensors_of_the_host(lib):
    d = mb.AttnDesc(2, 1, 64, 40, mb.F32)
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    ws = z(16, t=torch.uint8)
    cache = mb.alloc_paged_cache(d, mb.CACHE_I8, 4, 16, i(1, 2))
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        mb.HeadRopeCall(d, z(3, 2, 64), z(3, 1, 64), z(3, 2, 64), z(3, 1, 64), z(32))
    with pytest.raises(ValueError, match="k must be a GPU tensor"):
        mb.HeadRopeCall(d, None, z(3, 1, 64), None, z(3, 1, 64), z(32))
    with pytest.raises(ValueError, match="must not both be None"):
        mb.HeadRopeCall(d, None, None, None, None, z(32))
    with pytest.raises(ValueError, match="k_tree must be a GPU tensor"):
        mb.PagedWriteCall(d, cache, z(1, 3, 1, 64), z(1, 3, 1, 64), i(1))
    with pytest.raises(ValueError, match="k_pages must be a GPU tensor"):
        mb.PagedReadCall(d, cache, i(1), z(1, 1, 1, 40, 64), z(1, 1, 1, 40, 64))
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        mb.PagedAttentionCall(d, cache, z(1, 2, 64), i(1), ws, z(1, 2, 64))
    v = mb.VerifyDesc(50, mb.F32)
    with pytest.raises(ValueError, match="logits must be a GPU tensor"):
        mb.DraftVerifyCall(v, z(3, 50), i(3), z(3, t=torch.float64), z(1, t=torch.float64), i(1, 4), i(1), i(1), ws)


def test_pools_and_workspaces(lib):
    d = mb.AttnDesc(8, 2, 64, 40, mb.BF16)
    table = torch.zeros((3, 5), dtype=torch.int32)
    for code, held in ((mb.CACHE_PLAIN, torch.bfloat16), (mb.CACHE_I8, torch.int8), (mb.CACHE_E4M3, torch.float8_e4m3fn)):
        c = mb.alloc_paged_cache(d, code, 7, 32, table, n_layers=2)
        assert c.k_pages.shape == c.v_pages.shape == (2, 7, 2, 32, 64) and c.k_pages.dtype == held
        assert (c.k_scale is None) == (code == mb.CACHE_PLAIN) and (c.n_layers, c.max_entries) == (2, 160)
        assert mb.paged_attention_workspace_bytes(d, c, 3, 160) >= mb.paged_attention_workspace_bytes(d, c, 3, 10) > 0
        with pytest.raises(mb.MoeSpecError):
            mb.alloc_paged_attention_workspace(d, c, 3, 161)
    with pytest.raises(ValueError, match="unknown cache code"):
        mb.PagedCache(5, c.k_pages, c.v_pages, table).c(mb._Args(), d, 3)
    v = mb.VerifyDesc(50000, mb.BF16)
    assert mb.verify_workspace_bytes(v, 2, 30, True) >= 2 * mb.verify_workspace_bytes(v, 2, 30) > 0
    with pytest.raises(mb.MoeSpecError):
        mb.alloc_verify_workspace(mb.VerifyDesc(1, mb.F32), 1, 4)


# ---- the oracle against plain formulas

def test_oracle_rotation_is_a_rotation():
    rng = np.random.default_rng(0)
    x, place, freq = rng.standard_normal((5, 2, 8)), np.arange(5) * 3.0, np.array([1.0, 0.1, 0.01, 0.5])
    for inter in (False, True):
        out, _ = V.head_rope(x, None, place, freq, 8, inter)
        a, b = (slice(0, 8, 2), slice(1, 8, 2)) if inter else (slice(0, 4), slice(4, 8))
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * place[:, None] * freq)[:, None]
        assert np.allclose(out[..., a], z.real) and np.allclose(out[..., b], z.imag)
    out, _ = V.head_rope(x, np.arange(8.0), place, freq[:2], 4, norm=True, eps=0.5)
    want = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 0.5) * np.arange(8.0)
    assert np.allclose(out[..., 4:], want[..., 4:]) and np.allclose((out ** 2).sum(-1), (want ** 2).sum(-1))
    assert V.places([7, 0], [0, 3, 4], [A.ancestors([-1, 0, 0]), A.chain(1)]).tolist() == [7, 8, 8, 0]


def test_oracle_codes_against_torch():
    gen = torch.Generator().manual_seed(0)
    x = torch.randn((200, 64), generator=gen) * torch.exp2(torch.randint(-20, 20, (200, 1), generator=gen).float())
    codes, scale = V.codes_i8(x.double().numpy())
    assert np.abs(codes).max() == 127 and np.abs(codes * scale[:, None] - x.double().numpy()).max(1).max() > 0
    assert np.all(np.abs(codes * scale[:, None].astype(np.float64) - x.double().numpy()) <= scale[:, None] * (0.5 + 1e-5))
    values, scale = V.codes_e4m3(x.double().numpy())
    want = (x / torch.from_numpy(scale)[:, None]).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(values, want) and np.abs(values).max() <= 448 and np.abs(values).max() > 224
    assert np.all(np.log2(scale) == np.rint(np.log2(scale)))


def test_oracle_attention_against_torch():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 4, 8)), rng.standard_normal((2, 9, 8)), rng.standard_normal((2, 9, 8))
    out, lse, _, _ = V.attention(q, [k, k[:, :0]], [v, v[:, :0]], 0.3)
    kk, vv = (torch.from_numpy(t).repeat_interleave(2, dim=0) for t in (k, v))
    a = 0.3 * torch.einsum("hd,hnd->hn", torch.from_numpy(q[0]), kk)
    assert np.allclose(out[0], torch.einsum("hn,hnd->hd", a.softmax(1), vv)) and np.allclose(lse[0], torch.logsumexp(a, 1))
    assert not out[1].any() and np.all(np.isneginf(lse[1]))


def test_oracle_verification_keeps_the_target_distribution():
    """Exact: summed over a fine grid of the random numbers, what follows the root is distributed as the target."""
    p, q = np.log([0.5, 0.3, 0.2]), np.log([0.2, 0.2, 0.6])
    rows, n = np.tile(p, (3, 1)), 60
    grid = (np.arange(n) + 0.5) / n
    for draft in (None, np.tile(q, (3, 1))):
        seen = np.zeros(3)
        for x, px in enumerate(np.exp(q) if draft is not None else [1.0, 0.0, 0.0]):
            if px == 0:
                continue
            for u in grid:
                for w in grid:
                    path, token = V.verify(rows[:2], [0, x], A.chain(2), [0.0, u], w, 2, 1.0, None if draft is None else draft[:2])
                    seen[x if len(path) == 2 else token] += px / n ** 2
        assert np.allclose(seen, np.exp(p), atol=2.5 / n), seen
    # two children of one root, tokens 0 and 2: the second is judged by what the first has left
    seen = np.zeros(3)
    for u in grid:
        for u2 in grid:
            path, token = V.verify(rows, [0, 0, 2], A.ancestors([-1, 0, 0]), [0.0, u, u2], 0.25, 2)
            seen[{1: 0, 2: 2}[path[1]] if len(path) == 2 else token] += 1 / n ** 2
    assert np.allclose(seen, np.exp(p), atol=2.5 / n), seen


def test_oracle_verification_by_hand():
    rows = np.log(np.array([[0.1, 0.9], [0.6, 0.4], [0.5, 0.5]]))
    sees = A.ancestors([-1, 0, 1])
    assert V.verify(rows, [0, 1, 0], sees, [0, 0.89, 0.59], 0.49, 8) == ([0, 1, 2], 0)
    assert V.verify(rows, [0, 1, 0], sees, [0, 0.91, 0.59], 0.49, 8) == ([0], 0)
    assert V.verify(rows, [0, 1, 0], sees, [0, 0.89, 0.61], 0.0, 8) == ([0, 1], 1)
    assert V.verify(rows, [0, 1, 0], sees, [0, 0.89, 0.59], 0.49, 2) == ([0, 1], 0)  # cut: the accepted token follows
    assert V.verify(rows, [0, 1, 1], sees, [9, 9, 9], 0.99, 8, heat=0.0) == ([0, 1], 0)
