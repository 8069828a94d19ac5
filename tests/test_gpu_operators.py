"""The operators on a paged cache against their definitions in 64 bits (oracle/operators.py), at the sizes, layouts and
contents where they can go wrong.  Whatever no call may read -- positions behind a sequence's length, pages nobody owns --
holds NaN."""
import numpy as np
import pytest

from oracle import operators as plain

pytestmark = pytest.mark.gpu
PAGE = 64


@pytest.fixture(scope="module")
def bpd():
    import paper_1811_03115_b200 as b
    return b


def _round(x, dtype):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    return t.bfloat16().float().numpy() if dtype == "bf16" else t.numpy()


def _dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x))
    return t.to("cuda", torch.bfloat16 if dtype == "bf16" else t.dtype)


class Case:
    """A cache of ``layers`` layers with NaN wherever nothing was written, drafted nodes and their trees."""

    def __init__(self, seed, lens, nodes, heads, kv_heads, dim, dtype, layers=1, tree="random", live=None, spare=1):
        rng = self.rng = np.random.default_rng(seed)
        b = len(lens)
        self.lens, self.heads, self.kv_heads, self.dim, self.dtype, self.layers = np.asarray(lens, np.int32), heads, kv_heads, dim, dtype, layers
        ppr = max(1, -(-(int(max(lens)) + nodes) // PAGE))
        n_pages = b * ppr + spare
        self.table = rng.permutation(n_pages)[:b * ppr].reshape(b, ppr).astype(np.int32)
        shape = (layers, n_pages, PAGE, kv_heads, dim)
        self.k, self.v = np.full(shape, np.nan, np.float32), np.full(shape, np.nan, np.float32)
        for r, n in enumerate(lens):
            s = np.arange(n)
            for pool in (self.k, self.v):
                pool[:, self.table[r, s // PAGE], s % PAGE] = _round(rng.standard_normal((layers, n, kv_heads, dim)), dtype)
        self.q = _round(1.5 * rng.standard_normal((b, nodes, heads, dim)), dtype)
        self.k_new, self.v_new = (_round(rng.standard_normal((layers, b, nodes, kv_heads, dim)), dtype) for _ in range(2))
        t = np.arange(nodes)
        if tree == "chain":
            self.parents = np.tile(t - 1, (b, 1)).astype(np.int32)
        elif tree == "star":
            self.parents = np.full((b, nodes), -1, np.int32)
        else:
            self.parents = np.stack([np.maximum(t - 1 - rng.integers(0, 4, nodes), -1) for _ in range(b)]).astype(np.int32)
        self.nodes = np.full(b, nodes, np.int32) if live is None else np.asarray(live, np.int32)
        self.scale = dim ** -0.5

    def pools(self, layer=None):
        k, v = (self.k, self.v) if layer is None else (self.k[layer], self.v[layer])
        return _dev(k, self.dtype), _dev(v, self.dtype), _dev(self.table)

    def drafted(self, layer=0):
        return _dev(self.q, self.dtype), _dev(self.k_new[layer], self.dtype), _dev(self.v_new[layer], self.dtype)

    def weight_error(self):
        """Bound on the relative error of a softmax weight: the scores' (every step of 16 products may lose 2^-23 of the partial
        sum, which is at most sum |q||k|; the scale's rounding; log2(e) goes into it), the exponential's 2 units, the weight's
        16 (bf16) or 24 (fp32) bits, and the sum's, which is added up chunk by chunk."""
        keys = np.abs(np.nan_to_num(np.concatenate([self.k.reshape(-1, self.dim), self.k_new.reshape(-1, self.dim)], 0), posinf=0., neginf=0.)).max()
        score = self.scale * float(np.abs(np.nan_to_num(self.q, posinf=0., neginf=0.)).sum(-1).max()) * float(keys)
        chunks = max(self.lens) / 64 + 8
        return score * (self.dim / 16 + 4) * 2.0 ** -23, 2.0 ** -21 + (2.0 ** -17 if self.dtype == "bf16" else 2.0 ** -22) + 4 * chunks * 2.0 ** -24

    def check(self, got, want, want_lse, lse):
        score, rest = self.weight_error()
        far = np.nanmax(np.abs(want)) if want.size else 1.0
        # weights and their sum are both off by `score` and `rest`; values are below max |v|
        top = np.nanmax(np.abs(np.nan_to_num(np.concatenate([self.v.reshape(-1), self.v_new.reshape(-1)]), posinf=0., neginf=0.)))
        half = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -23
        tol = 2 * (score + rest) * max(top, far) + half * np.abs(want)
        got = got.double().cpu().numpy()
        assert got.shape == want.shape and not np.isnan(got).any()
        assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) - tol).max())
        if lse is not None:
            lse = lse.double().cpu().numpy()
            assert np.array_equal(np.isinf(lse), np.isinf(want_lse)) and (lse[np.isinf(lse)] < 0).all()
            seen = ~np.isinf(want_lse)
            assert (np.abs(lse - want_lse)[seen] <= (score + rest + 2.0 ** -22 * np.abs(want_lse[seen]) + 2.0 ** -21)).all()


# lengths 0 and 1, page edges, tiles of 16, 32 and 64 rows and several of them, groups that do not divide a tile, trees that
# span several words, rows with fewer nodes than others and with none
TREES = [
    ([0], 1, 1, 1, 16, "chain", None), ([1], 1, 4, 4, 64, "chain", None), ([63, 64, 65], 1, 8, 2, 128, "chain", None),
    ([130, 0, 200], 10, 4, 4, 64, "chain", [10, 3, 0]), ([100, 7], 13, 6, 2, 32, "random", [13, 5]), ([1000], 5, 24, 2, 64, "random", None),
    ([300, 64], 33, 2, 2, 128, "random", [33, 1]), ([700, 5], 64, 4, 2, 64, "random", [64, 50]), ([90], 65, 3, 1, 16, "random", None),
    ([129], 200, 2, 1, 64, "random", None), ([20], 256, 1, 1, 32, "chain", None), ([64], 100, 2, 2, 128, "star", None),
    ([2500, 1, 640, 64], 3, 16, 1, 128, "random", [3, 1, 2, 3]), ([40] * 130, 2, 2, 1, 16, "chain", None),
    ([1500], 1, 1, 1, 64, "chain", None), ([1500, 30], 3, 1, 1, 128, "chain", None), ([900], 5, 3, 1, 16, "random", None), ([2000, 1], 70, 4, 2, 128, "random", [70, 9]),
    ([4100, 300], 20, 4, 2, 64, "random", [20, 7]), ([4160, 0], 13, 3, 1, 128, "chain", [13, 2]), ([600, 448, 1], 256, 2, 2, 64, "random", [256, 130, 3]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,tree,live", TREES)
def test_tree_attention(bpd, lens, nodes, heads, kv_heads, dim, tree, live, dtype):
    c = Case(nodes * dim + len(lens), lens, nodes, heads, kv_heads, dim, dtype, tree=tree, live=live)
    want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
    out, lse = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents), None if live is None else _dev(c.nodes), want_lse=True)
    c.check(out, want, want_lse, lse)
    again = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents), None if live is None else _dev(c.nodes))
    assert bool((again == out).all())                       # the same call gives the same bits


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tree_attention_of_slices_of_one_projection(bpd, dtype):
    import torch
    c = Case(3, [70, 130], 5, 4, 2, 64, dtype)
    width = (4 + 2 * 2) * 64
    fused = torch.full((2, 5, width + 16), float("nan"), device="cuda", dtype=_dev(c.q, dtype).dtype)
    q, k, v = c.drafted()
    fused[..., :256], fused[..., 256:384], fused[..., 384:512] = q.flatten(2), k.flatten(2), v.flatten(2)
    parts = fused[..., :256].unflatten(2, (4, 64)), fused[..., 256:384].unflatten(2, (2, 64)), fused[..., 384:512].unflatten(2, (2, 64))
    got = bpd.bpd_op_tree_attention(*parts, *c.pools(0), _dev(c.lens), _dev(c.parents), scale=0.3)
    assert bool((got == bpd.bpd_op_tree_attention(q, k, v, *c.pools(0), _dev(c.lens), _dev(c.parents), scale=0.3)).all())
    c.scale = 0.3
    c.check(got, *plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, 0.3), None)


# siblings hold infinities and NaN: only their own lines may see them
@pytest.mark.parametrize("dtype,dim,nodes,length", [("bf16", 64, 9, 10), ("fp32", 64, 9, 10), ("bf16", 128, 40, 0), ("fp32", 16, 20, 10), ("bf16", 64, 9, 500),
                                                    ("bf16", 128, 70, 1000), ("bf16", 64, 100, 700), ("fp32", 32, 70, 600)])
def test_values_that_are_no_numbers_stay_in_their_line(bpd, dtype, dim, nodes, length):
    c = Case(5, [length, 0], nodes, 2, 1, dim, dtype, tree="star")
    c.parents[:, 3] = 1
    c.parents[:, 4] = 3
    bad = [2, 5, nodes - 1]
    c.k_new[:, :, 2], c.v_new[:, :, 2] = np.nan, np.inf
    c.v_new[:, :, 5, :, ::3] = np.nan
    c.k_new[:, :, nodes - 1], c.v_new[:, :, nodes - 1, :, 1] = np.inf, -np.inf
    want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
    out, lse = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents), want_lse=True)
    fine = [t for t in range(nodes) if t not in bad]
    c.check(out[:, fine], want[:, fine], want_lse[:, fine], lse[:, fine])
    assert bool(out[:, 2].isnan().all()) and bool(out[:, 5, :, ::3].isnan().all()) and bool(out[:, 5, :, 1::3].isfinite().all())


# and whoever does see them has no finite output there, even with a weight that is 0 in 32 bits
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim,nodes,length", [(64, 9, 10), (128, 20, 0), (16, 40, 30), (64, 70, 300), (128, 100, 900)])
def test_values_that_are_no_numbers_show_whatever_their_weight(bpd, dim, nodes, length, dtype):
    c = Case(15, [length, 5], nodes, 2, 1, dim, dtype, tree="chain")
    c.q[..., 3], c.k_new[..., 3] = 8, 8                      # scores of 64 times the scale and more, against -64 times 32: weights of 0
    c.k_new[:, :, 2, :, 3] = -2048
    c.v_new[:, :, 2, :, ::2], c.v_new[:, :, 2, :, 1] = np.inf, np.nan
    out = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents))
    bad = np.zeros(dim, bool)
    bad[::2], bad[1] = True, True
    fine = out.isfinite().cpu().numpy()
    assert not fine[:, 2:][..., bad].any() and fine[:, :2].all() and fine[..., ~bad].all()


# the largest numbers of the type likewise; what sees them comes out as they are, times the weight
@pytest.mark.parametrize("dim,nodes,length", [(64, 9, 10), (16, 20, 10), (128, 40, 0), (32, 70, 600)])
def test_largest_values_stay_in_their_line(bpd, dim, nodes, length):
    c = Case(13, [length, 0], nodes, 2, 1, dim, "fp32", tree="star")
    bad, far = [2, nodes - 1], np.finfo(np.float32)
    c.v_new[:, :, 2, :, ::3], c.v_new[:, :, nodes - 1, :, 1] = far.min, np.float32(3.397e38)
    want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
    out, lse = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents), want_lse=True)
    c.v_new = np.where(np.abs(c.v_new) < 100, c.v_new, 0)    # check's tolerance goes by the largest value that a row sees
    fine = [t for t in range(nodes) if t not in bad]
    c.check(out[:, fine], want[:, fine], want_lse[:, fine], lse[:, fine])
    rest = sum(c.weight_error()) * 2 + 2.0 ** -22
    for t, cols in ((2, slice(0, None, 3)), (nodes - 1, slice(1, 2))):
        assert (np.abs(out[:, t, :, cols].double().cpu().numpy() / want[:, t, :, cols] - 1) <= rest).all()


# Infinities and the largest numbers that every row sees, in 32 bits: keys of weight 0 for them, a query's element that meets zeros,
# values of both kinds.  Tiles of 16, 32 and 64 rows, whole and in runs, selected pages.
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,select", [([70, 130], 1, 2, 2, 64, 0), ([900, 64], 5, 2, 1, 16, 0), ([2000], 20, 2, 2, 128, 0),
                                                                  ([700, 100], 40, 2, 1, 32, 0), ([300], 70, 3, 1, 64, 0), ([1500], 3, 4, 2, 64, 30)])
def test_tree_attention_of_the_largest_numbers(bpd, lens, nodes, heads, kv_heads, dim, select):
    import torch
    c = Case(17, lens, nodes, heads, kv_heads, dim, "fp32")
    far = np.finfo(np.float32)
    c.q[..., 3], c.q[..., 4] = np.abs(c.q[..., 3]) + 0.25, -np.abs(c.q[..., 4]) - 0.25
    c.k[..., 5], c.k_new[..., 5], c.q[:, nodes // 2, :, 5] = 0, 0, far.max
    for r, n in enumerate(lens):
        at = lambda s: (0, c.table[r, s // PAGE], s % PAGE)
        for s, d, x in ((0, 3, -np.inf), (9, 3, far.min), (18, 4, far.max), (n // 2, 4, np.inf), (n // 2 + 1, 3, np.float32(-3.397e38)), (n - 1, 4, far.max)):
            c.k[at(s) + (slice(None), d)] = x
        for s, d, x in ((1, 7, np.inf), (n // 2 + 2, 8, far.min), (n - 2, 9, np.float32(3.397e38)), (2, 10, -np.inf)):
            c.v[at(s) + (slice(None), d)] = x
    c.k_new[:, :, 0, :, 4] = far.max
    d = c.drafted() + c.pools(0)
    if select:
        means = np.zeros((len(lens),) + c.table.shape[1:] + (kv_heads, dim), np.float32)
        want, want_lse, _ = plain.page_attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, means, c.lens, c.parents, select, c.nodes, c.scale)
        out, lse = bpd.bpd_op_page_attention(*d, _dev(means), _dev(c.lens), _dev(c.parents), select, want_lse=True)
    else:
        want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
        out, lse = bpd.bpd_op_tree_attention(*d, _dev(c.lens), _dev(c.parents), want_lse=True)
    c.q, c.k, c.v, c.k_new = (np.where(np.isnan(x) | (np.abs(x) < 100), x, 0) for x in (c.q, c.k, c.v, c.k_new))    # what check's tolerance goes by
    rest = sum(c.weight_error()) * 2 + 2.0 ** -22
    odd = np.zeros(dim, bool)
    odd[7:11] = True
    got = out.double().cpu().numpy()
    assert np.array_equal(got[..., [7, 10]], want[..., [7, 10]]) and np.isinf(want[..., [7, 10]]).all()
    assert (np.abs(got[..., 8:10] / want[..., 8:10] - 1) <= rest).all() and (np.abs(want[..., 8:10]) > 1e20).all()
    c.check(out[..., torch.from_numpy(~odd).cuda()], want[..., ~odd], want_lse, lse)


# queries that are no numbers, as rows of padding may hold: theirs are the only outputs that show it
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim", [([70, 5], 3, 2, 2, 64), ([900, 1300], 9, 4, 2, 64), ([900, 0], 40, 2, 1, 128), ([700, 900], 70, 2, 1, 64), ([500], 5, 2, 1, 16)])
def test_queries_that_are_no_numbers(bpd, lens, nodes, heads, kv_heads, dim, dtype):
    c = Case(19, lens, nodes, heads, kv_heads, dim, dtype)
    want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
    _, k_new, v_new = c.drafted()
    q = c.q.copy()
    q[:, nodes // 2], q[:, nodes - 1, :, 1] = np.nan, np.nan
    out, lse = bpd.bpd_op_tree_attention(_dev(q, dtype), k_new, v_new, *c.pools(0), _dev(c.lens), _dev(c.parents), want_lse=True)
    bad = sorted({nodes // 2, nodes - 1})
    fine = [t for t in range(nodes) if t not in bad]
    c.check(out[:, fine], want[:, fine], want_lse[:, fine], lse[:, fine])
    assert bool(out[:, bad].isnan().all()) and bool(lse[:, bad].isnan().all())


# pages outside the pool, parents that do not lie before their node, lengths and node counts outside their ranges
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_of_device_arrays_are_not_trusted(bpd, dtype):
    c = Case(6, [200, 130, 90], 6, 4, 2, 32, dtype, spare=3)
    c.table[0, 1], c.table[1, 2], c.table[2, 0] = -1, len(c.k[0]), 2 ** 31 - 1
    c.parents[0] = [5, 1, 7, -3, 2, 2]
    out, lse = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents), want_lse=True)
    c.check(out, *plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale), lse)
    many = Case(7, [500, 450, 700], 40, 4, 2, 64, dtype, spare=2)
    many.table[0, 2], many.table[1, 7], many.table[2, 0] = -7, len(many.k[0]), 2 ** 31 - 1
    out, lse = bpd.bpd_op_tree_attention(*many.drafted(), *many.pools(0), _dev(many.lens), _dev(many.parents), want_lse=True)
    many.check(out, *plain.attention(many.q, many.k_new[0], many.v_new[0], many.k[0], many.v[0], many.table, many.lens, many.parents, many.nodes, many.scale), lse)
    lens, nodes = np.array([-5, 2 ** 31 - 1, 90], np.int32), np.array([99, -2, 2 ** 31 - 1], np.int32)
    c.k[:], c.v[:] = np.nan_to_num(c.k), np.nan_to_num(c.v)
    out, lse = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(lens), _dev(c.parents), _dev(nodes), want_lse=True)
    c.nodes, c.lens = np.array([6, 0, 6], np.int32), np.array([0, 256, 90], np.int32)
    c.check(out, *plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale), lse)


PAGED = [
    ([0], 1, 1, 1, 16, 1, None), ([64], 1, 2, 2, 64, 1, None), ([63], 2, 4, 2, 64, 3, None), ([1000, 130], 3, 8, 2, 128, 4, [3, 2]),
    ([700, 64, 65, 5], 2, 20, 1, 64, 5, [2, 0, 1, 2]), ([2000], 1, 40, 2, 32, 7, None), ([5000], 4, 4, 4, 16, 30, None), ([640], 70, 2, 1, 64, 2, [70]),
    ([2000, 700], 1, 1, 1, 64, 9, None), ([1500], 2, 3, 1, 128, 8, None),
    # more pages than a thread's or a lane's registers hold keys of
    ([1500, 90], 2, 80, 1, 64, 9, None), ([5000], 1, 40, 1, 128, 70, None), ([900, 64], 70, 66, 1, 64, 8, [70, 3]),
    ([160003], 1, 2, 1, 16, 9, None), ([70003, 160000], 5, 1, 1, 16, 40, [5, 3]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,select,live", PAGED)
def test_page_attention(bpd, lens, nodes, heads, kv_heads, dim, select, live, dtype):
    import torch
    c = Case(nodes + dim + len(lens), lens, nodes, heads, kv_heads, dim, dtype, live=live)
    means = plain.page_means(c.k[0], c.table, c.lens)
    k, v, table = c.pools(0)
    held = torch.full((1,) + means.shape, float("nan"), device="cuda")
    half = np.maximum(c.lens // 2, 0).astype(np.int32)
    bpd.bpd_op_page_means(k[None], table, _dev(np.zeros_like(half)), _dev(half), held)          # in two steps, as a cache grows
    bpd.bpd_op_page_means(k[None], table, _dev(half), _dev(c.lens), held)
    got = held[0].cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(means))
    np.testing.assert_allclose(np.nan_to_num(got), np.nan_to_num(means), rtol=2.0 ** -23)
    means = got
    want, want_lse, pages = plain.page_attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, means, c.lens, c.parents, select, c.nodes, c.scale)
    out, lse, chosen = bpd.bpd_op_page_attention(*c.drafted(), k, v, table, held[0], _dev(c.lens), _dev(c.parents), select,
                                                 None if live is None else _dev(c.nodes), want_lse=True, want_pages=True)
    assert np.array_equal(chosen.cpu().numpy(), pages)
    c.check(out, want, want_lse, lse)


def test_page_selection_orders_ties_and_no_numbers(bpd):
    c = Case(9, [64 * 9 + 3], 1, 2, 1, 64, "fp32")
    means = np.zeros((1, 10, 1, 64), np.float32)
    means[0, :9, 0, 0] = [1, 2, np.nan, 2, -np.inf, 2, 0, -0.0, 2]
    c.q[:] = 0
    c.q[0, 0, :, 0] = [0.25, 0.75]
    for select, want in ((2, [1, 3]), (5, [0, 1, 3, 5, 8]), (7, [0, 1, 3, 5, 6, 7, 8])):
        # a product of 0 and -inf is no number either: page 4's scores are NaN where the query is 0, and go with page 2
        pages = bpd.bpd_op_page_attention(*c.drafted(), *c.pools(0), _dev(means), _dev(c.lens), _dev(c.parents), select, want_pages=True)[1]
        assert pages[0, 0, 0].tolist() == want
    assert bpd.bpd_op_page_attention(*c.drafted(), *c.pools(0), _dev(means), _dev(c.lens), _dev(c.parents), 8, want_pages=True)[1][0, 0, 0].tolist() == [0, 1, 3, 4, 5, 6, 7, 8]
    assert bpd.bpd_op_page_attention(*c.drafted(), *c.pools(0), _dev(means), _dev(c.lens), _dev(c.parents), 12, want_pages=True)[1][0, 0, 0].tolist() == list(range(9)) + [-1] * 3


@pytest.mark.parametrize("layers,lens,nodes,kv_heads,dim,dtype,eos", [(1, [0], 1, 1, 16, "bf16", -1), (3, [62, 5, 127], 9, 2, 64, "fp32", -1),
                                                                      (2, [60] * 40, 33, 4, 32, "bf16", 1), (6, [10, 128], 256, 8, 128, "bf16", -1)])
def test_tree_commit(bpd, layers, lens, nodes, kv_heads, dim, dtype, eos):
    b = len(lens)
    c = Case(layers * nodes, lens, nodes, kv_heads, kv_heads, dim, dtype, layers=layers, live=None if nodes == 1 else [nodes - (r % 3) for r in range(b)])
    tokens, top1, last = (c.rng.integers(0, 2, s).astype(np.int32) for s in ((b, nodes), (b, nodes), b))
    tokens[0], top1[0], last[0] = 0, 0, 0                    # a long walk
    want = plain.commit(c.k_new, c.v_new, c.k, c.v, c.table, c.lens, c.parents, tokens, top1, last, c.nodes, eos)
    k, v, table = c.pools()
    got = bpd.bpd_op_tree_commit(_dev(c.k_new, dtype), _dev(c.v_new, dtype), k, v, table, _dev(c.lens), _dev(c.parents), _dev(tokens), _dev(top1), _dev(last),
                                 _dev(c.nodes), eos_id=eos)
    for x, y in zip(got + (k, v), want):
        assert np.array_equal(x.float().cpu().numpy(), np.asarray(y, np.float32), equal_nan=True)


def test_tree_commit_stops_where_the_cache_is_full(bpd):
    c = Case(4, [125, 128, 120], 8, 1, 1, 16, "fp32", tree="chain")
    c.table = c.table[:, :2].copy()
    c.table[2, 1] = -1                                       # that row's second page is missing: its entries are not written
    zeros = np.zeros((3, 8), np.int32)
    k, v, table = c.pools()
    got = bpd.bpd_op_tree_commit(_dev(c.k_new), _dev(c.v_new), k, v, table, _dev(c.lens), _dev(c.parents), _dev(zeros), _dev(zeros), _dev(zeros[:, 0]))
    assert got[0].tolist() == [128, 128, 128] and got[1].tolist() == [3, 0, 8]
    want = plain.commit(c.k_new, c.v_new, c.k, c.v, c.table, c.lens, c.parents, zeros, zeros, zeros[:, 0], c.nodes)
    assert np.array_equal(k.cpu().numpy(), want[4], equal_nan=True) and np.array_equal(v.cpu().numpy(), want[5], equal_nan=True)
    bad = bpd.bpd_op_tree_commit(_dev(c.k_new), _dev(c.v_new), k, v, table, _dev(np.array([-1, 129, 128], np.int32)), _dev(c.parents), _dev(zeros), _dev(zeros),
                                 _dev(zeros[:, 0]))
    assert bad[1].tolist() == [0, 0, 0] and np.array_equal(k.cpu().numpy(), want[4], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim", [([0], 1, 1, 1, 16), ([63, 64, 1], 3, 4, 2, 64), ([600, 0, 1100], 5, 8, 2, 128), ([130], 40, 6, 2, 32),
                                                           ([513], 20, 16, 2, 16)])
def test_cache_weights(bpd, lens, nodes, heads, kv_heads, dim, dtype):
    c = Case(dim + nodes, lens, nodes, heads, kv_heads, dim, dtype, tree="chain")
    b, cap = len(lens), c.table.shape[1] * PAGE
    accepted = np.array([min(nodes, 1 + 2 * r + nodes // 2) for r in range(b)], np.int32)
    if b > 2:
        accepted[2] = 0
    # the path's nodes in ascending order, their keys in the cache as the commit leaves them
    path = np.full((b, nodes), -1, np.int32)
    for r in range(b):
        path[r, :accepted[r]] = np.sort(c.rng.permutation(nodes)[:accepted[r]])
        for i in range(accepted[r]):
            s = lens[r] + i
            c.k[0, c.table[r, s // PAGE], s % PAGE] = c.k_new[0, r, path[r, i]]
    lse = np.full((b, nodes, heads), np.nan, np.float32)
    for r in range(b):
        for i in range(accepted[r]):
            for g in range(heads):
                keys = plain.cached(c.k[0][:, :, g * kv_heads // heads], c.table[r], range(lens[r] + i + 1))
                lse[r, path[r, i], g] = plain.softmax_row(c.q[r, path[r, i], g].astype(np.float64), keys, keys, c.scale)[1]
    weights = c.rng.random((b, kv_heads, cap)).astype(np.float32)
    positions = c.rng.integers(0, 1000, (b, kv_heads, cap)).astype(np.int32)
    seen = np.arange(b).astype(np.int32) * 1000 + 7
    want_w, want_p = plain.cache_weights(c.q, lse, path, accepted, c.k[0], c.table, c.lens, seen, weights, positions, c.scale)
    k, _, table = c.pools(0)
    got_w, got_p = _dev(weights), _dev(positions)
    bpd.bpd_op_cache_weights(_dev(c.q, dtype), _dev(lse), _dev(path), _dev(accepted), k, table, _dev(c.lens), _dev(seen), got_w, got_p)
    assert np.array_equal(got_p.cpu().numpy(), want_p)
    score, _ = c.weight_error()
    # a weight's exponent is off by the score's error, and by the rounding of the difference to lse; the exponential by 2 units, the
    # sums by one rounding for each of up to 64 rows
    off = score + 2.0 ** -24 * np.nanmax(np.abs(lse)) + 2.0 ** -21 + 64 * 2.0 ** -24
    got = got_w.double().cpu().numpy()
    assert (np.abs(got - want_w) <= off * (want_w + 1e-30) + 2.0 ** -23 * want_w).all()
    untouched = np.ones_like(weights, bool)
    for r in range(b):
        untouched[r, :, :lens[r] + accepted[r] if accepted[r] else 0] = False
    assert np.array_equal(got_w.cpu().numpy()[untouched], weights[untouched])


# a length outside the cache comes back as the other calls read it
def test_tree_commit_clamps_lengths(bpd):
    c = Case(4, [100, 100, 100, 100], 8, 1, 1, 16, "fp32", tree="chain")
    c.table = c.table[:, :2].copy()
    zeros = np.zeros((4, 8), np.int32)
    k, v, table = c.pools()
    before = k.clone(), v.clone()
    got = bpd.bpd_op_tree_commit(_dev(c.k_new), _dev(c.v_new), k, v, table, _dev(np.array([-1, 129, -2 ** 31, 2 ** 31 - 1], np.int32)), _dev(c.parents),
                                 _dev(zeros), _dev(zeros), _dev(zeros[:, 0]))
    assert got[0].tolist() == [0, 128, 0, 128] and got[1].tolist() == [0] * 4 and bool((got[2] == -1).all())
    assert all(bool(((x == y) | (x.isnan() & y.isnan())).all()) for x, y in zip((k, v), before))


class WeightsCase(Case):
    """A path of accepted nodes whose keys are in the cache, as a commit leaves them; lse in 64 bits, rounded."""

    def __init__(self, seed, lens, accepted, nodes, heads, kv_heads, dim, dtype, change=lambda c: None):
        super().__init__(seed, lens, nodes, heads, kv_heads, dim, dtype, tree="chain")
        b, cap = len(lens), self.table.shape[1] * PAGE
        self.accepted = np.asarray(accepted, np.int32)
        self.path = np.full((b, nodes), -1, np.int32)
        for r in range(b):
            self.path[r, :accepted[r]] = np.sort(self.rng.permutation(nodes)[:accepted[r]])
            for i in range(accepted[r]):
                s = lens[r] + i
                self.k[0, self.table[r, s // PAGE], s % PAGE] = self.k_new[0, r, self.path[r, i]]
        change(self)
        self.q = _round(self.q, dtype)                       # both sides get what the type holds
        self.lse = np.full((b, nodes, heads), np.nan, np.float32)
        for r in range(b):
            for i in range(accepted[r]):
                for g in range(heads):
                    keys = plain.cached(self.k[0][:, :, g * kv_heads // heads], self.table[r], range(lens[r] + i + 1))
                    self.lse[r, self.path[r, i], g] = plain.softmax_row(self.q[r, self.path[r, i], g].astype(np.float64), keys, keys, self.scale)[1]
        self.weights = self.rng.random((b, kv_heads, cap)).astype(np.float32)
        self.positions = self.rng.integers(0, 1000, (b, kv_heads, cap)).astype(np.int32)
        self.seen = np.arange(b).astype(np.int32) * 1000 + 7

    def check_weights(self, bpd):
        want_w, want_p = plain.cache_weights(self.q, self.lse, self.path, self.accepted, self.k[0], self.table, self.lens, self.seen, self.weights,
                                             self.positions, self.scale)
        k, _, table = self.pools(0)
        got_w, got_p = _dev(self.weights), _dev(self.positions)
        bpd.bpd_op_cache_weights(_dev(self.q, self.dtype), _dev(self.lse), _dev(self.path), _dev(self.accepted), k, table, _dev(self.lens), _dev(self.seen),
                                 got_w, got_p)
        assert np.array_equal(got_p.cpu().numpy(), want_p)
        # as in test_cache_weights: the score's error, the difference to lse, 2 units of the exponential, a rounding for each row of a sum
        rows = int(self.accepted.max()) * self.heads // self.kv_heads
        off = self.key_error() + 2.0 ** -24 * np.nanmax(np.abs(self.lse)) + 2.0 ** -21 + (rows + 2) * 2.0 ** -24
        got = got_w.double().cpu().numpy()
        assert not np.isnan(got).any()
        assert (np.abs(got - want_w) <= off * (want_w + 1e-30) + 2.0 ** -23 * want_w).all()

    def key_error(self):
        """weight_error's first part over keys of ordinary size (those beyond give a weight of 0 or are set by hand)."""
        keys = np.abs(np.concatenate([self.k.reshape(-1), self.k_new.reshape(-1)]))
        keys = keys[keys < 100].max()
        q = np.where(np.abs(self.q) < 100, np.abs(self.q), 0)
        return self.scale * float(q.sum(-1).max()) * float(keys) * (self.dim / 16 + 4) * 2.0 ** -23


# A cached key with an infinite element whose products are all -inf has weight 0, whatever the number of rows (they are padded
# to eight)
@pytest.mark.parametrize("lens,accepted,nodes,heads,kv_heads,dim", [([100], [1], 1, 1, 1, 64), ([130, 70], [3, 2], 4, 6, 2, 128), ([200], [8], 9, 2, 2, 32),
                                                                    ([90], [5], 5, 3, 1, 16), ([300], [9], 12, 8, 1, 64)])
def test_cache_weights_of_infinite_keys(bpd, lens, accepted, nodes, heads, kv_heads, dim):
    def change(c):
        c.q[..., 3] = np.abs(c.q[..., 3]) + 0.25
        for r, n in enumerate(lens):
            for s in (0, 17, n - 1):
                c.k[0, c.table[r, s // PAGE], s % PAGE, :, 3] = -np.inf
    WeightsCase(dim, lens, accepted, nodes, heads, kv_heads, dim, "bf16", change).check_weights(bpd)


# The same in 32 bits, with the largest finite numbers too: among keys whose weight is 0 for them, and in a query against zeros
@pytest.mark.parametrize("lens,accepted,nodes,heads,kv_heads,dim", [([100], [1], 1, 1, 1, 64), ([130, 70], [3, 2], 4, 6, 2, 128), ([200], [8], 9, 2, 2, 32),
                                                                    ([90], [5], 5, 3, 1, 16), ([300], [9], 12, 8, 1, 64)])
def test_cache_weights_of_the_largest_numbers(bpd, lens, accepted, nodes, heads, kv_heads, dim):
    far = np.finfo(np.float32)

    def change(c):
        c.q[..., 3], c.q[..., 4] = np.abs(c.q[..., 3]) + 0.25, -np.abs(c.q[..., 4]) - 0.25
        c.k[..., 5], c.k_new[..., 5] = 0, 0
        for r, n in enumerate(lens):
            c.q[r, c.path[r, accepted[r] - 1], :, 5] = far.max
            for s, d, x in ((0, 3, -np.inf), (9, 3, far.min), (18, 4, far.max), (n // 2, 4, np.inf), (n // 2 + 1, 3, np.float32(-3.397e38)), (n - 1, 4, far.max)):
                c.k[0, c.table[r, s // PAGE], s % PAGE, :, d] = x
    WeightsCase(dim, lens, accepted, nodes, heads, kv_heads, dim, "fp32", change).check_weights(bpd)


EVICT = [(1, [1], 1, 16, 1, 0, "bf16"), (2, [65, 10, 64], 2, 32, 20, 5, "fp32"), (1, [522], 4, 64, 512, 64, "fp32"), (3, [700, 300], 2, 128, 100, 100, "bf16"),
         (1, [1500, 1], 3, 64, 1, 0, "bf16"), (2, [3000], 2, 16, 2999, 7, "bf16"), (1, [1024, 513, 512], 1, 32, 512, 0, "fp32"),
         # more slots than registers hold keys of
         (1, [9000, 100], 1, 16, 700, 33, "bf16"), (1, [20000, 17001], 1, 16, 9000, 50, "fp32")]


@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
@pytest.mark.parametrize("layers,lens,kv_heads,dim,budget,recent,dtype", EVICT)
def test_cache_evict(bpd, layers, lens, kv_heads, dim, budget, recent, dtype, kind):
    c = Case(budget + dim, lens, 1, kv_heads, kv_heads, dim, dtype, layers=layers)
    b, cap = len(lens), c.table.shape[1] * PAGE
    shape = (layers, b, kv_heads, cap)
    weights = c.rng.random(shape).astype(np.float32)
    if kind == "ties":
        weights = np.floor(weights * 3).astype(np.float32) - 1                  # -1, 0, 1
        weights[..., ::5] = -0.0
    elif kind == "odd":
        weights[c.rng.random(shape) < 0.3] = np.nan
        weights[c.rng.random(shape) < 0.1] = -np.inf
        weights[c.rng.random(shape) < 0.1] = np.inf
    positions = np.stack([c.rng.permutation(cap) for _ in range(layers * b * kv_heads)]).reshape(shape).astype(np.int32)
    seen = np.array([cap - 3 * r for r in range(b)], np.int32)
    want = plain.evict(weights, positions, c.k, c.v, c.table, c.lens, seen, budget, recent)
    k, v, table = c.pools()
    w, p = _dev(weights), _dev(positions)
    got = bpd.bpd_op_cache_evict(w, p, k, v, table, _dev(c.lens), _dev(seen), budget, recent)
    for x, y in zip((got, w, p, k, v), want):
        assert np.array_equal(x.float().cpu().numpy(), np.asarray(y, np.float32), equal_nan=True)


# ---------------------------------------------------------------------- runs of many turns, other layouts, the ends of the ranges
def _far(seed, lens, nodes, heads, kv_heads, dim, dtype):
    """Tensors of a long cache on the device, and bounds as Case.check takes them."""
    import torch
    gen = torch.Generator("cuda").manual_seed(seed)
    dt, b = (torch.bfloat16 if dtype == "bf16" else torch.float32), len(lens)
    ppr = -(-(max(lens) + nodes) // PAGE)
    t = {n: torch.empty(s, dtype=dt, device="cuda").normal_(generator=gen) for n, s in
         (("k", (b * ppr, PAGE, kv_heads, dim)), ("v", (b * ppr, PAGE, kv_heads, dim)), ("q", (b, nodes, heads, dim)), ("k_new", (b, nodes, kv_heads, dim)),
          ("v_new", (b, nodes, kv_heads, dim)))}
    t["table"] = torch.randperm(b * ppr, generator=gen, device="cuda").view(b, ppr).int()
    t["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    t["parents"] = (torch.arange(nodes, device="cuda") - 1).expand(b, nodes).int().contiguous()
    return t


# A CTA's run of more chunks than it looks up pages for at once (64): 444 CTAs share 2 x 8 x 3750 of them, and 296 share more than
# 64 each in the others; tiles of 16, 32, 64 and 128 rows
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim", [([239963, 200001], 3, 8, 8, 16), ([239963, 200001], 4, 48, 8, 16), ([100000, 160001], 9, 24, 4, 32),
                                                           ([150003] * 3, 40, 8, 4, 64)])
def test_tree_attention_of_long_runs(bpd, lens, nodes, heads, kv_heads, dim, dtype):
    import torch
    t = _far(41, lens, nodes, heads, kv_heads, dim, dtype)
    out, lse = bpd.bpd_op_tree_attention(t["q"], t["k_new"], t["v_new"], t["k"], t["v"], t["table"], t["lens"], t["parents"], want_lse=True)
    scale, g = dim ** -0.5, heads // kv_heads
    # as Case.weight_error
    score = scale * float(t["q"].double().abs().sum(-1).max()) * float(torch.stack([t[n].abs().max() for n in ("k", "k_new")]).max()) * (dim / 16 + 4) * 2.0 ** -23
    rest = 2.0 ** -21 + (2.0 ** -17 if dtype == "bf16" else 2.0 ** -22) + 4 * (max(lens) / 64 + 8) * 2.0 ** -24
    top = float(torch.stack([t[n].abs().max() for n in ("v", "v_new")]).max())
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    tree = torch.ones(nodes, nodes, dtype=torch.bool, device="cuda").tril()
    for b, n in enumerate(lens):
        pages = t["table"][b].long()
        for h in range(kv_heads):
            keys, values = (torch.cat([t[p][pages, :, h].reshape(-1, dim)[:n], t[p + "_new"][b, :, h]]).double() for p in ("k", "v"))
            q = t["q"][b, :, h * g:(h + 1) * g].double()
            s = q @ keys.T * scale
            s[..., n:].masked_fill_(~tree[:, None, :], -torch.inf)
            want, want_lse = torch.softmax(s, -1) @ values, torch.logsumexp(s, -1)
            got = out[b, :, h * g:(h + 1) * g].double()
            assert bool(((got - want).abs() <= 2 * (score + rest) * top + half * want.abs()).all())
            assert bool(((lse[b, :, h * g:(h + 1) * g].double() - want_lse).abs() <= score + rest + 2.0 ** -22 * want_lse.abs() + 2.0 ** -21).all())


# Warps that take several tiles of a page run, runs that go on with another key head and another sequence, sequences that accepted
# nothing among them: 2700 pages for 296 CTAs
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv_heads,heads,dim", [(2, 2, 64), (2, 6, 16), (1, 2, 128)])
def test_cache_weights_of_long_runs(bpd, kv_heads, heads, dim, dtype):
    few = 1 if kv_heads == 2 else 2
    lens = [6400, 6399 * few, 1, 0, 12801 * few, 5000, 64, 9000 * few, 63, 7777, 12800 * few, 4095, 3]
    accepted = [3, 1, 4, 2, 1, 0, 4, 2, 0, 4, 3, 1, 0]
    WeightsCase(51, lens, accepted, 4, heads, kv_heads, dim, dtype).check_weights(bpd)


# more columns than a CTA's threads take at once
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kv_heads,dim", [(32, 128), (65, 64), (300, 16)])
def test_page_means_of_wide_rows(bpd, kv_heads, dim, dtype):
    import torch
    c = Case(53, [200, 64], 1, kv_heads, kv_heads, dim, dtype, layers=2)
    k, _, table = c.pools()
    held = torch.full((2,) + c.table.shape + (kv_heads, dim), float("nan"), device="cuda")
    bpd.bpd_op_page_means(k, table, _dev(np.zeros(2, np.int32)), _dev(c.lens), held)
    for layer in range(2):
        want, got = plain.page_means(c.k[layer], c.table, c.lens), held[layer].cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        np.testing.assert_allclose(np.nan_to_num(got), np.nan_to_num(want), rtol=2.0 ** -23)


def _fused(*parts):
    """The tensors [..., heads, dim] as slices of one row each, with NaN between and behind them."""
    import torch
    rows = [p.flatten(-2) for p in parts]
    row = torch.full(rows[0].shape[:-1] + (sum(r.shape[-1] + 16 for r in rows) + 24,), float("nan"), device="cuda", dtype=rows[0].dtype)
    at, out = 8, []
    for p, r in zip(parts, rows):
        row[..., at:at + r.shape[-1]] = r
        out.append(row[..., at:at + r.shape[-1]].unflatten(-1, p.shape[-2:]))
        at += r.shape[-1] + 16
    assert row.shape[:-1].numel() == 1 or not any(o.is_contiguous() for o in out)
    return out


# every kernel that reads rows of drafted nodes, with rows further apart than they are wide: whole tiles and runs, few and many rows,
# the selection for one node and for several
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,select", [([70], 1, 4, 4, 32, 0), ([900, 1300], 5, 4, 2, 64, 0), ([900, 10], 33, 4, 2, 128, 0), ([700, 900], 70, 2, 1, 64, 0),
                                                                  ([800, 1], 70, 4, 2, 128, 0), ([1500, 700], 1, 4, 2, 64, 9), ([1500], 6, 80, 1, 128, 9), ([2000, 65], 5, 6, 3, 16, 4)])
def test_rows_further_apart_than_wide(bpd, lens, nodes, heads, kv_heads, dim, select, dtype):
    import torch
    c = Case(55, lens, nodes, heads, kv_heads, dim, dtype, live=[nodes] + [max(1, nodes - 2)] * (len(lens) - 1))
    k, v, table = c.pools(0)
    rest = (_dev(c.lens), _dev(c.parents))
    means = torch.zeros((1,) + c.table.shape + (kv_heads, dim), device="cuda")
    bpd.bpd_op_page_means(k[None], table, torch.zeros_like(rest[0]), rest[0], means)

    def call(q, k_new, v_new):
        if select:
            return bpd.bpd_op_page_attention(q, k_new, v_new, k, v, table, means[0], *rest, select, nodes=_dev(c.nodes), want_lse=True, want_pages=True)
        return bpd.bpd_op_tree_attention(q, k_new, v_new, k, v, table, *rest, nodes=_dev(c.nodes), want_lse=True)
    for x, y in zip(call(*c.drafted()), call(*_fused(*c.drafted()))):
        assert bool((x == y).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_commit_and_weights_of_rows_further_apart_than_wide(bpd, dtype):
    c = WeightsCase(57, [130, 62, 700], [3, 5, 2], 7, 6, 2, 64, dtype)
    k, _, table = c.pools(0)

    def weights(q):
        w, p = _dev(c.weights), _dev(c.positions)
        bpd.bpd_op_cache_weights(q, _dev(c.lse), _dev(c.path), _dev(c.accepted), k, table, _dev(c.lens), _dev(c.seen), w, p)
        return w, p
    q = _dev(c.q, dtype)
    for x, y in zip(weights(q), weights(_fused(q)[0])):
        assert bool((x == y).all())
    layers = Case(58, [130, 62, 5], 7, 2, 2, 64, dtype, layers=3, tree="chain")
    zeros = np.zeros((3, 7), np.int32)

    def commit(k_new, v_new):
        k, v, table = layers.pools()
        got = bpd.bpd_op_tree_commit(k_new, v_new, k, v, table, _dev(layers.lens), _dev(layers.parents), _dev(zeros), _dev(zeros), _dev(zeros[:, 0]))
        return got + (k, v)
    rows = _dev(layers.k_new, dtype), _dev(layers.v_new, dtype)
    for x, y in zip(commit(*rows), commit(*_fused(*rows))):
        assert bool(((x == y) | (x.isnan() & y.isnan())).all())


# rows that share the pages of a common beginning, each with an open page of its own
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("nodes,dim", [(3, 64), (70, 128)])
def test_sequences_that_share_pages(bpd, nodes, dim, dtype):
    c = Case(59, [700, 660, 643], nodes, 2, 1, dim, dtype)
    c.table[1, :10] = c.table[2, :10] = c.table[0, :10]
    out, lse = bpd.bpd_op_tree_attention(*c.drafted(), *c.pools(0), _dev(c.lens), _dev(c.parents), want_lse=True)
    c.check(out, *plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale), lse)


# a batch of nothing but padding; far more heads to a key head than a tile has rows; many sequences; many key heads
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,select", [([70, 5], 3, 2, 2, 64, 0), ([700, 5], 3, 2, 2, 64, 0), ([700, 5], 40, 4, 2, 128, 0), ([700, 5], 3, 2, 2, 64, 4)])
def test_a_batch_of_padding(bpd, lens, nodes, heads, kv_heads, dim, select, dtype):
    import torch
    c = Case(61, lens, nodes, heads, kv_heads, dim, dtype)
    none = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    args = c.drafted() + c.pools(0)
    if select:
        means = torch.zeros(c.table.shape + (kv_heads, dim), device="cuda")
        out, lse, pages = bpd.bpd_op_page_attention(*args, means, _dev(c.lens), _dev(c.parents), select, nodes=none, want_lse=True, want_pages=True)
        assert bool((pages == -1).all())
    else:
        out, lse = bpd.bpd_op_tree_attention(*args, _dev(c.lens), _dev(c.parents), nodes=none, want_lse=True)
    assert bool((out == 0).all()) and bool(lse.isneginf().all())
    k, v, table = c.pools()
    zeros = torch.zeros(len(lens), nodes, dtype=torch.int32, device="cuda")
    got = bpd.bpd_op_tree_commit(_dev(c.k_new, dtype), _dev(c.v_new, dtype), k, v, table, _dev(c.lens), _dev(c.parents), zeros, zeros, none + 9, nodes=none)
    assert got[0].tolist() == lens and not bool(got[1].any()) and bool((got[2] == -1).all()) and bool((got[3] == 9).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,select", [([300], 2, 300, 1, 64, 0), ([900], 1, 300, 1, 128, 5), ([500, 3], 2, 200, 1, 16, 3), ([3] * 700, 1, 1, 1, 16, 0),
                                                                  ([2] * 699 + [900], 2, 2, 1, 32, 0), ([70], 1, 1024, 1024, 16, 0), ([450], 2, 600, 300, 32, 3)])
def test_many_heads_and_many_sequences(bpd, lens, nodes, heads, kv_heads, dim, select, dtype):
    import torch
    c = Case(63, lens, nodes, heads, kv_heads, dim, dtype)
    k, v, table = c.pools(0)
    if select:
        held = torch.zeros((1,) + c.table.shape + (kv_heads, dim), device="cuda")
        bpd.bpd_op_page_means(k[None], table, _dev(np.zeros_like(c.lens)), _dev(c.lens), held)
        want, want_lse, pages = plain.page_attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, held[0].cpu().numpy(), c.lens, c.parents, select, c.nodes, c.scale)
        out, lse, chosen = bpd.bpd_op_page_attention(*c.drafted(), k, v, table, held[0], _dev(c.lens), _dev(c.parents), select, want_lse=True, want_pages=True)
        assert np.array_equal(chosen.cpu().numpy(), pages)
    else:
        want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
        out, lse = bpd.bpd_op_tree_attention(*c.drafted(), k, v, table, _dev(c.lens), _dev(c.parents), want_lse=True)
    c.check(out, want, want_lse, lse)


# what a race would show: the same call fifty times, with other work on the device between; many short runs that end and begin
# inside tiles, and long ones
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens,nodes,heads,kv_heads,dim,select", [([900], 70, 66, 1, 64, 8), ([900], 60, 80, 1, 128, 9), ([3000, 100, 2000], 40, 4, 1, 128, 0),
                                                                  ([2500] * 5, 64, 4, 2, 64, 0), ([5000], 5, 8, 2, 64, 20), ([700] * 20, 16, 2, 2, 32, 0)])
def test_the_same_call_gives_the_same_bits(bpd, lens, nodes, heads, kv_heads, dim, select, dtype):
    import torch
    c = Case(31, lens, nodes, heads, kv_heads, dim, dtype)
    q, k_new, v_new = c.drafted()
    k, v, table = c.pools(0)
    lens_d, parents = _dev(c.lens), _dev(c.parents)
    means = torch.zeros((1,) + c.table.shape + (kv_heads, dim), device="cuda")
    bpd.bpd_op_page_means(k[None], table, torch.zeros_like(lens_d), lens_d, means)

    def call():
        if select:
            return bpd.bpd_op_page_attention(q, k_new, v_new, k, v, table, means[0], lens_d, parents, select)
        return bpd.bpd_op_tree_attention(q, k_new, v_new, k, v, table, lens_d, parents)
    first, noise = call(), torch.empty(1 << 22, device="cuda")
    same = []
    for i in range(50):
        if i % 3 == 0:
            noise.normal_()
        same.append((call() == first).all())
    assert bool(torch.stack(same).all())


# calls side by side on two streams, each with a scratch and outputs of its own
def test_two_streams_do_not_meet(bpd):
    import torch
    cases = [Case(21, [700, 90, 1500], 6, 4, 2, 64, "bf16"), Case(22, [1200], 40, 4, 1, 128, "bf16"), Case(23, [900, 10], 5, 2, 1, 32, "fp32")]
    args = [c.drafted() + c.pools(0) + (_dev(c.lens), _dev(c.parents)) for c in cases]
    alone = [bpd.bpd_op_tree_attention(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    got = [[] for _ in args]
    for _ in range(20):
        for a, s, g in zip(args, streams, got):
            with torch.cuda.stream(s):
                g.append(bpd.bpd_op_tree_attention(*a))
    torch.cuda.synchronize()
    for want, g in zip(alone, got):
        assert all(bool((x == want).all()) for x in g)
    bpd.bpd_op_status()                                      # no wait has expired


# a wait that expires is reported once, and what follows is right
def test_an_expired_wait_is_reported(bpd):
    c = Case(25, [700, 90], 40, 4, 2, 128, "bf16")
    args = c.drafted() + c.pools(0) + (_dev(c.lens), _dev(c.parents))
    bpd.bpd_op_status()
    first = bpd.bpd_op_tree_attention(*args)
    bpd.bpd_debug_op_wait_timeout(2000)
    again = bpd.bpd_op_tree_attention(*args)
    with pytest.raises(bpd.BpdError, match="expired"):
        bpd.bpd_op_status()
    bpd.bpd_op_status()
    assert bool((first == again).all())


# a program's step: attention over the cache and the tree, commit, weights, eviction, and the next step's attention over what is
# left, eagerly and as one captured graph replayed on another stream
def _steps(bpd, c, state, budget):
    out, lse = bpd.bpd_op_tree_attention(state["q"], state["k_new"][0], state["v_new"][0], state["k"][0], state["v"][0], state["table"], state["lens"],
                                         state["parents"], want_lse=True)
    lens, accepted, path, following = bpd.bpd_op_tree_commit(state["k_new"], state["v_new"], state["k"], state["v"], state["table"], state["lens"],
                                                             state["parents"], state["tokens"], state["top1"], state["last"])
    bpd.bpd_op_cache_weights(state["q"], lse, path, accepted, state["k"][0], state["table"], state["lens"], state["seen"], state["weights"][0],
                             state["positions"][0])
    left = bpd.bpd_op_cache_evict(state["weights"], state["positions"], state["k"], state["v"], state["table"], lens, state["seen"] + accepted, budget, 8)
    after, _ = bpd.bpd_op_tree_attention(state["q"], state["k_new"][0], state["v_new"][0], state["k"][0], state["v"][0], state["table"], left, state["parents"],
                                         want_lse=True)
    state["means"].zero_()
    bpd.bpd_op_page_means(state["k"], state["table"], state["zero"], left, state["means"])
    paged, pages = bpd.bpd_op_page_attention(state["q"], state["k_new"][0], state["v_new"][0], state["k"][0], state["v"][0], state["table"], state["means"][0],
                                             left, state["parents"], 1, want_pages=True)
    return out, lse, lens, accepted, path, following, left, after, paged, pages


@pytest.mark.parametrize("captured", [False, True])
def test_a_step_of_all_operators(bpd, captured):
    import torch
    budget = 130
    c = Case(11, [150, 131, 40], 7, 4, 2, 64, "fp32", live=None)
    b, cap = 3, c.table.shape[1] * PAGE
    tokens, top1, last = np.zeros((b, 7), np.int32), np.zeros((b, 7), np.int32), np.zeros(b, np.int32)
    weights, seen = c.rng.random((1, b, 2, cap)).astype(np.float32), c.lens.copy()
    positions = np.broadcast_to(np.arange(cap, dtype=np.int32), (1, b, 2, cap)).copy()
    host = {"k_new": c.k_new, "v_new": c.v_new, "k": c.k, "v": c.v, "table": c.table, "lens": c.lens, "parents": c.parents, "tokens": tokens, "top1": top1,
            "last": last, "weights": weights, "positions": positions, "seen": seen, "q": c.q, "zero": np.zeros(b, np.int32),
            "means": np.zeros((1,) + c.table.shape + (2, 64), np.float32)}
    state = {n: _dev(x) for n, x in host.items()}
    if captured:
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream):
            _steps(bpd, c, state, budget)                  # loads the kernels
            with torch.cuda.graph(graph, stream=stream):
                got = _steps(bpd, c, state, budget)
        torch.cuda.synchronize()
        for n, x in host.items():
            state[n].copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            graph.replay()
        torch.cuda.synchronize()
    else:
        got = _steps(bpd, c, state, budget)
    out, lse, lens, accepted, path, following, left, after, paged, pages = got
    want, want_lse = plain.attention(c.q, c.k_new[0], c.v_new[0], c.k[0], c.v[0], c.table, c.lens, c.parents, c.nodes, c.scale)
    c.check(out, want, want_lse, lse)
    new = plain.commit(c.k_new, c.v_new, c.k, c.v, c.table, c.lens, c.parents, tokens, top1, last, c.nodes)
    for x, y in zip((lens, accepted, path, following), new):
        assert np.array_equal(x.cpu().numpy(), y)
    assert accepted.min() >= 1
    k, v = new[4], new[5]
    w, p = plain.cache_weights(c.q, want_lse, new[2], new[1], k[0], c.table, c.lens, seen, weights[0], positions[0], c.scale)
    # the library's weights are these to rounding; drawn weights lie far enough apart that the same entries stay
    lefts, w, p, k, v = plain.evict(w[None], p[None], k, v, c.table, new[0], seen + new[1], budget, 8)
    assert np.array_equal(left.cpu().numpy(), lefts) and lefts.tolist()[:2] == [130, 130]
    assert np.array_equal(state["positions"].cpu().numpy(), p)
    assert np.array_equal(state["k"].cpu().numpy(), k, equal_nan=True) and np.array_equal(state["v"].cpu().numpy(), v, equal_nan=True)
    c.k, c.v, c.lens = k, v, lefts
    c.check(after, *plain.attention(c.q, c.k_new[0], c.v_new[0], k[0], v[0], c.table, lefts, c.parents, c.nodes, c.scale), None)
    means = state["means"][0].cpu().numpy()
    far = plain.page_attention(c.q, c.k_new[0], c.v_new[0], k[0], v[0], c.table, means, lefts, c.parents, 1, c.nodes, c.scale)
    assert np.array_equal(pages.cpu().numpy(), far[2])
    c.check(paged, far[0], far[1], None)
