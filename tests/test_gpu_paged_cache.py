"""Writing to pages and reading them back: codes and scales bit for bit, what is dropped, what stays as it was."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as V
from paper_2602_16052_amd import binding as mb
from attention_common import CODE, TORCH, f64, i32
from serving_common import KIND, table, values64

pytestmark = pytest.mark.gpu


class Case:
    """Trees of L layers behind caches of their own, and a pool filled with 1 (scales with 2)."""

    def __init__(self, dtype, code, Hk, D, lens, trees, page, layers=1, fused=False, pad=0, seed=0, room=40, rows=None):
        rng, gen = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
        self.off = np.concatenate([[0], np.cumsum(trees)])
        M, dt = int(self.off[-1]) + pad, TORCH[dtype]
        randn = lambda *s: (torch.randn(s, generator=gen, device="cuda") * 3).to(dt)  # noqa: E731
        if fused:
            qkv = randn(layers, M, 3 * Hk, D)
            self.k, self.v = qkv[:, :, Hk:2 * Hk], qkv[:, :, 2 * Hk:]
        else:
            self.k, self.v = randn(layers, M, Hk, D), randn(layers, M, Hk, D)
        self.rows, n = table([x + room for x in lens], page, rng) if rows is None else rows
        self.desc = mb.AttnDesc(Hk, Hk, D, max(lens) + room, CODE[dtype])
        self.cache = mb.alloc_paged_cache(self.desc, KIND[code], n, page, torch.from_numpy(self.rows).cuda(), layers)
        self.code, self.lens, self.page, self.trees = code, lens, page, trees
        for t in (self.cache.k_pages, self.cache.v_pages):
            t.copy_(torch.ones(t.shape, device="cuda"))
        for t in (self.cache.k_scale, self.cache.v_scale):
            if t is not None:
                t.fill_(2.0)
        self.args = dict(tree_off=i32(self.off), max_tree=max(max(trees), 1))

    def write(self, paths=None, max_path=None):
        kw = {}
        if paths is not None:
            n = max_path or max(len(p) for p in paths)
            at = np.full((len(paths), n), 2 ** 30)
            for s, p in enumerate(paths):
                at[s, :len(p)] = p
            kw = dict(path=i32(at), n_path=i32([len(p) for p in paths]))
        return mb.moespec_paged_write(self.desc, self.cache, self.k, self.v, i32(self.lens), **kw, **self.args)

    def expected(self, paths):
        """(codes' values, scales) of the whole pool as they must be, for k and v."""
        c, res = self.cache, []
        for x in (self.k, self.v):
            pages, scales = np.ones(c.k_pages.shape), np.full(c.k_pages.shape[:-1], 2.0, dtype=np.float32)
            src = f64(x)
            for s, p in enumerate(paths):
                for i, t in enumerate(p):
                    e = self.lens[s] + i
                    if e >= self.rows.shape[1] * self.page:
                        continue
                    at = self.rows[s][e // self.page]
                    if not 0 <= at < pages.shape[1]:
                        continue
                    row = src[:, self.off[s] + t] if 0 <= t < self.trees[s] else np.zeros((src.shape[0],) + src.shape[2:])
                    if self.code == "plain":
                        pages[:, at, :, e % self.page] = row
                    else:
                        pages[:, at, :, e % self.page], scales[:, at, :, e % self.page] = \
                            (V.codes_i8 if self.code == "i8" else V.codes_e4m3)(row)
            res.append((pages, scales))
        return res

    def check(self, paths):
        c = self.cache
        for (pages, scales), got, got_scale in zip(self.expected(paths), (c.k_pages, c.v_pages), (c.k_scale, c.v_scale)):
            assert np.array_equal(values64(got), pages, equal_nan=True)
            if got_scale is not None:
                assert np.array_equal(got_scale.cpu().numpy(), scales, equal_nan=True)


def whole(trees):
    return [list(range(n)) for n in trees]


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("code", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_whole_trees_by_type_code_and_head_size(dtype, code, D):
    c = Case(dtype, code, 3, D, [5, 0, 31], [20, 0, 7], 16, seed=D)
    new = c.write()
    assert new.tolist() == [25, 0, 38]
    c.check(whole(c.trees))


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages(page):
    c = Case("bf16", "i8", 1, 64, [page - 3, page, 2 * page - 1], [9, 40, 2], page, seed=page)
    c.write()
    c.check(whole(c.trees))


@pytest.mark.parametrize("code", ["plain", "i8", "e4m3"])
def test_paths_of_several_layers_out_of_a_projection(code):
    """Places in any order, the same one twice, places outside of the tree, an empty path, rows of no sequence behind the last."""
    paths = [[0, 3, 9, 9, 2], [], [0], [1, 5, -1, 99]]
    c = Case("bf16", code, 2, 128, [17, 3, 100, 0], [10, 4, 1, 6], 32, layers=3, fused=True, pad=5, seed=1)
    assert c.write(paths, max_path=7).tolist() == [22, 3, 101, 4]
    c.check([[t if 0 <= t < n else -1 for t in p] for p, n in zip(paths, c.trees)])


def test_long_prompts():
    c = Case("bf16", "e4m3", 2, 64, [0, 3], [700, 1300], 64, seed=2, room=1400)
    c.write()
    c.check(whole(c.trees))


def test_what_does_not_fit_is_dropped():
    rows = np.array([[2, 0], [1, 5], [-1, 3]], dtype=np.int32), 5  # page 5 is outside of the pool
    c = Case("bf16", "i8", 1, 64, [28, 10, 14], [10, 10, 6], 16, rows=rows, seed=3)
    assert c.write().tolist() == [32, 20, 20]
    c.check(whole(c.trees))


def test_lengths_out_of_range():
    c = Case("f32", "plain", 1, 64, [0, 0], [3, 3], 16, seed=4)
    cap = c.rows.shape[1] * 16
    got = mb.moespec_paged_write(c.desc, c.cache, c.k, c.v, i32([-9, 2 ** 31 - 1]), path=i32([[0, 1], [0, 1]]), n_path=i32([2 ** 30, -4]),
                                 **c.args)
    assert got.tolist() == [2, cap]
    c.check([[0, 1], []])


@pytest.mark.parametrize("code", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_the_borders_of_the_codes(dtype, code):
    """Zeros, the smallest and largest values, a single large one, ties of the rounding, powers of two and their neighbours, rows that are not
    finite."""
    big, tiny = float(torch.finfo(TORCH[dtype]).max), float(torch.finfo(TORCH[dtype]).tiny)
    c = Case(dtype, code, 1, 64, [0], [16], 16, seed=5)
    x = c.k[0, :, 0]
    x[0] = 0
    x[1] = tiny
    x[2] = big
    x[3] = 0
    x[3, 7] = -1.0
    x[4] = torch.arange(64, device="cuda") * 2.0 - 63.0  # amax 63: steps of 63 / 127
    x[5] = (torch.arange(64, device="cuda") - 32) * 0.5 + 0.25
    x[5, 0] = 127.0
    x[6] = 448.0
    x[7, 0] = 448.0 * 4 * (1 + 2.0 ** -7)
    x[8] = torch.exp2(-torch.arange(64, device="cuda").float())  # down to what e4m3 cannot hold
    x[9] = torch.exp2(-torch.arange(64, device="cuda").float()) * 1.5
    x[10, 3] = float("inf")
    x[11, 4] = float("nan")
    x[12, 5] = -float("inf")
    x[13] = tiny / 8 if dtype == "f32" else tiny
    x[14] = torch.linspace(-1, 1, 64, device="cuda")
    x[15] = torch.linspace(-447, 449, 64, device="cuda")
    c.v.copy_(c.k.flip(1))
    c.write()
    c.check(whole(c.trees))
    d, n = c.desc, i32([16])
    k, _ = mb.moespec_paged_read(d, c.cache, n)
    k = k[0, 0, 0]
    assert torch.isnan(k[10:13]).all() and torch.count_nonzero(k[0]) == 0


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("code", ["plain", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_reading(dtype, code, D):
    """All entries, entries from a place on, others left alone, entries without a page as zeros, lengths past the bound."""
    c = Case(dtype, code, 2, D, [0, 0, 0], [45, 1, 20], 16, layers=2, seed=D + 1, room=60)
    c.write()
    rows = c.rows.copy()
    rows[2, 0] = -1
    c.cache.page_table.copy_(torch.from_numpy(rows))
    cap, first = c.desc.capacity, [0, 1, 5]
    for start in (None, first):
        k, v = (torch.full((2, 3, 2, cap, D), 9.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
        mb.moespec_paged_read(c.desc, c.cache, i32([45, 1, 2 ** 30]), k, v, first=None if start is None else i32(start), max_len=20 if start else 45)
        for got, (pages, scales) in zip((k, v), c.expected(whole(c.trees))):
            want = np.full((2, 3, 2, cap, D), 9.0)
            for s, n in enumerate([20, 1, 20] if start else [45, 1, 45]):
                for e in range(start[s] if start else 0, n):
                    if s == 2 and e < 16:
                        want[:, s, :, e] = 0
                        continue
                    at = rows[s][e // 16]
                    x = pages[:, at, :, e % 16]
                    if code != "plain":  # the product in fp32, then the type
                        x = (x.astype(np.float32) * scales[:, at, :, e % 16, None])
                    want[:, s, :, e] = f64(torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[dtype]))
            assert np.array_equal(f64(got), want)


def test_reading_nothing():
    c = Case("bf16", "i8", 1, 64, [0], [5], 16)
    k, v = mb.moespec_paged_read(c.desc, c.cache, i32([5]), max_len=0)
    assert torch.count_nonzero(k) == 0 and torch.count_nonzero(v) == 0
    k, _ = mb.moespec_paged_read(c.desc, c.cache, i32([3]), first=i32([3]))
    assert torch.count_nonzero(k) == 0


def test_offsets_behind_32_bits():
    n = (1 << 32) // (256 * 256) + 3
    rows = np.array([[0, n - 1]], dtype=np.int32), n
    c = Case("bf16", "i8", 1, 256, [250], [20], 256, rows=rows)
    c.write()
    k, v = mb.moespec_paged_read(c.desc, c.cache, i32([270]), first=i32([250]))
    for got, src in ((k, c.k), (v, c.v)):
        codes, scale = V.codes_i8(f64(src)[0, :, 0])
        want = codes.astype(np.float32) * scale[:, None]
        assert np.array_equal(f64(got[0, 0, 0, 250:270]), f64(torch.from_numpy(want).to(torch.bfloat16)))
    assert int((c.cache.k_pages[0, 1:n - 1] != 1).sum()) == 0


def test_a_captured_write_follows_lengths_and_paths():
    c = Case("bf16", "e4m3", 2, 128, [3, 30], [8, 8], 16, layers=2, seed=7, room=90)
    lens, path, n_path, new = i32(c.lens), i32([[0, 1, 2], [0, 4, 5]]), i32([1, 3]), i32([0, 0])
    call = mb.PagedWriteCall(c.desc, c.cache, c.k, c.v, lens, path, n_path, new, **c.args)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    want = []
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            call()
        start, steps = list(c.lens), [([0], [0, 4, 5]), ([0, 6, 7], []), ([2, 2], [1])]
        for a, b in steps:
            at = np.zeros((2, 3))
            at[0, :len(a)], at[1, :len(b)] = a, b
            path.copy_(i32(at)), n_path.copy_(i32([len(a), len(b)]))
            graph.replay()
            stream.synchronize()
            want.append((a, b))
            lens.copy_(new)
    assert lens.tolist() == [start[0] + 6, start[1] + 4]
    c.check([sum((w[0] for w in want), []), sum((w[1] for w in want), [])])
