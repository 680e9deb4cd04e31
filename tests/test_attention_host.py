"""The calls around a verification step's attention without a GPU: argument checks and workspace sizes through the C ABI under
sanitizers (tests/host_checks_attention.c), the binding's checks of tensors, and the oracle against plain formulas."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import attention_oracle as A
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
    exe = str(tmp_path / "host_checks_attention")
    cc = subprocess.run([clang, "-std=c11", "-O1", "-g", "-Wall", "-Wextra", "-pedantic", "-Werror",
                         "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
                         "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host_checks_attention.c"),
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


def test_binding_reports_sizes_and_errors(lib):
    d = mb.AttnDesc(8, 2, 64, 100, mb.BF16)
    assert mb.check_attn_desc(d) == mb.OK and d.c().scale == 0.125
    assert mb.check_attn_desc(mb.AttnDesc(8, 3, 64, 100, mb.BF16)) == mb.ERR_INVALID_ARG
    assert mb.check_attn_desc(mb.AttnDesc(8, 2, 72, 100, mb.BF16)) == mb.ERR_UNSUPPORTED_SHAPE
    with pytest.raises(mb.MoeSpecError):
        mb.alloc_attn_workspace(d, 1, 8, 9, 100)
    with pytest.raises(mb.MoeSpecError):
        mb.alloc_evict_workspace(d, 1, 1, 0)


def test_binding_refuses_tensors_of_the_host(lib):
    """Every entry point names the first tensor that is not on a GPU, before it crosses the boundary."""
    d = mb.AttnDesc(2, 1, 64, 10, mb.F32)
    z = lambda *s, t=torch.float32: torch.zeros(s, dtype=t)  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    ws = z(16, t=torch.uint8)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        mb.TreeAttentionCall(d, z(3, 2, 64), z(3, 1, 64), z(3, 1, 64), z(1, 1, 10, 64), z(1, 1, 10, 64), i(1), ws, z(3, 2, 64))
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        mb.CacheWeightsCall(d, z(3, 2, 64), z(3, 1, 64), z(1, 1, 10, 64), i(1), z(3, 2), ws, z(1, 1, 10))
    with pytest.raises(ValueError, match="k_tree must be a GPU tensor"):
        mb.CacheCommitCall(d, z(1, 3, 1, 64), z(1, 3, 1, 64), i(1, 2), i(1), z(1, 1, 1, 10, 64), z(1, 1, 1, 10, 64), i(1))
    with pytest.raises(ValueError, match="k_cache must be a GPU tensor"):
        mb.CacheEvictCall(d, z(1, 1, 1, 10, 64), z(1, 1, 1, 10, 64), z(1, 1, 1, 10), i(1), 4, 1, z(1, 1, 1, 4, 64),
                          z(1, 1, 1, 4, 64), z(1, 1, 1, 4), ws)
    with pytest.raises(ValueError, match="y must be a GPU tensor"):
        mb.BlockNormCall(mb.LayerDesc(64, 1, 1, 64, mb.F32, False), z(3, 64), None, None, z(3, 64))


# ---- the oracle

def test_oracle_attention_is_softmax_attention():
    rng = np.random.default_rng(0)
    T, H, Hk, D, n = 5, 4, 2, 8, 7
    q, kt, vt = rng.normal(size=(T, H, D)), rng.normal(size=(T, Hk, D)), rng.normal(size=(T, Hk, D))
    kc, vc = rng.normal(size=(1, Hk, 9, D)), rng.normal(size=(1, Hk, 9, D))
    sees = A.ancestors([-1, 0, 0, 2, -1])
    out, lse, bound, spread = A.attention(q, kt, vt, kc, vc, [n], [0, T], [sees], 0.3)
    for h in range(H):
        k = np.concatenate([kc[0, h // 2, :n], kt[:, h // 2]])
        v = np.concatenate([vc[0, h // 2, :n], vt[:, h // 2]])
        mask = np.concatenate([np.ones((T, n), bool), sees], axis=1)
        ref = torch.nn.functional.scaled_dot_product_attention(
            torch.tensor(q[None, :, h]), torch.tensor(k[None]), torch.tensor(v[None]), torch.tensor(mask[None]), scale=0.3)[0]
        assert np.allclose(out[:, h], ref.numpy(), rtol=1e-12, atol=1e-14)
        a = np.where(mask, 0.3 * q[:, h] @ k.T, -np.inf)
        assert np.allclose(lse[:, h], np.log(np.exp(a).sum(axis=1)))
    assert np.all(np.abs(out) <= bound + 1e-15) and np.all(spread > 0)


def test_oracle_weights_are_the_columns_of_the_softmax():
    rng = np.random.default_rng(1)
    T, H, D, n = 4, 2, 8, 6
    q, kt, kc = rng.normal(size=(T, H, D)), rng.normal(size=(T, 1, D)), rng.normal(size=(1, 1, 8, D))
    sees = A.chain(T)
    vt, vc = np.zeros_like(kt), np.zeros_like(kc)
    lse = A.attention(q, kt, vt, kc, vc, [n], [0, T], [sees], 0.5)[1]
    rw = np.array([1.0, 0.5, 0.0, 2.0])
    w_in = rng.random((1, 1, 8))
    cw, tw, _, _ = A.weights(q, kt, kc, [n], [0, T], [sees], 0.5, lse, rw, w_in, 0.25)
    assert np.isclose(cw[0, 0, :n].sum() - 0.25 * w_in[0, 0, :n].sum() + tw.sum(), H * rw.sum())
    assert np.all(cw[0, 0, n:] == 0)


def test_oracle_eviction_and_masks_by_hand():
    assert list(A.kept_entries(np.array([5.0, 1, 5, 0, 9, 2]), 6, 4, 1)) == [0, 2, 4, 5]
    assert list(A.kept_entries(np.array([1.0, 1, 1, 1, 1]), 5, 3, 1)) == [0, 1, 4]
    assert list(A.kept_entries(np.array([np.nan, 0.0, np.nan, -np.inf]), 4, 2, 0)) == [1, 3]
    assert list(A.kept_entries(np.array([3.0, 2, 1]), 3, 3, 0)) == [0, 1, 2]
    words = A.pack([A.ancestors([-1, 0])], 3, 33, fill=1)
    assert words.shape == (3, 2) and words[0, 0] & 3 == 1 and words[1, 0] & 3 == 3 and words[2, 0] == -1


def test_oracle_block_norm_by_hand():
    y, res = np.array([[3.0, 4.0]]), np.array([[1.0, -1.0]])
    r, x, _ = A.block_norm(y, res, True, np.array([2.0, 1.0]), np.array([0.0]), True, 2.0, None, 0.0)
    rms = np.sqrt(12.5)
    assert np.allclose(r, [[1 + 2 * 0.5 * 2 * 3 / rms, -1 + 2 * 0.5 * 4 / rms]])
    assert np.allclose((x * x).mean(), 1.0)
