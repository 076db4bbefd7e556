"""shard_tree_attention and shard_tree_accept (include/shard.h) against plain
implementations in 64 bits.

Bound on an attention output, with A = sum_j p_j |v_j| over the visible entries
(p the exact softmax), c the count of them and half(t) = finfo(t).eps / 2:
  half(out) |o|         the output's rounding, or half the smallest subnormal
  half(kv) A            the weights' rounding to the cache's type before the
                        product with V (32-bit queries: two parts, half(kv)^2)
  2 D A                 D = the largest error of a score: (d + 2) 2^-24 of the sum
                        S of |q k| scale for 32-bit sums, 32-bit queries cut to two
                        parts (half(kv)^2 of S, or half the smallest subnormal
                        each); weights and their sum have it once each
  c 2^-22 A             exp and sums in 32 bits (c additions of half a step, or
                        four steps of exp where that is more: max(c, 4) 2^-24)
  c 2^-31 max |v|       a weight that fp16 holds as a subnormal, relative to the
                        largest weight times 2^6
"""
import numpy as np
import pytest
import torch

import paper_2608_19147_gb300 as pkg

pytestmark = pytest.mark.gpu
TYPES = {"f32": (torch.float32, pkg.SHARD_F32), "f16": (torch.float16, pkg.SHARD_F16), "bf16": (torch.bfloat16, pkg.SHARD_BF16)}
NAN = float("nan")


def trees(n, kind, gen):
    """parents of trees of n[b] nodes: a chain, random, or a star of nodes without a parent"""
    out = []
    for k in n:
        for i in range(k):
            out.append(-1 if i == 0 or kind == "star" else i - 1 if kind == "chain" else int(gen.integers(-1 if i % 7 == 6 else 0, i)))
    return out


class Case:
    """A batch with everything that no node may read filled with NaN."""

    def __init__(self, n, lens, heads, kv_heads, d, q="f16", kv="f16", out=None, kind="random", holes=0.0, by_entry=False, mask=True,
                 cap=None, pad=0, seed=0, extra_nodes=2):
        g = np.random.default_rng(seed)
        t = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.lens, self.heads, self.kv_heads, self.d = n, lens, heads, kv_heads, d
        self.q_type, self.kv_type, self.out_type = q, kv, out or q
        B, N = len(n), sum(n) + extra_nodes
        self.B, self.N = B, N
        self.cap = cap or max(a + b for a, b in zip(n, lens)) + 3
        self.start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.parents = np.array(trees(n, kind, g) + [-1] * extra_nodes, dtype=np.int32)
        self.q = torch.randn(N, heads * d + 8 * pad, generator=t, device="cuda").to(TYPES[q][0])
        shape = (B, self.cap, kv_heads, d) if by_entry else (B, kv_heads, self.cap, d)
        self.k_at = torch.randn(shape, generator=t, device="cuda").to(TYPES[kv][0])
        self.v_at = torch.randn(shape, generator=t, device="cuda").to(TYPES[kv][0])
        st = self.k_at.stride()
        self.strides = (st[0], st[2], st[1]) if by_entry else (st[0], st[1], st[2])
        self.k, self.v = (x.transpose(1, 2) if by_entry else x for x in (self.k_at, self.v_at))
        self.mask = (g.random((B, self.cap)) >= holes).astype(np.uint8) if mask else None
        for b in range(B):  # what nobody sees
            P = lens[b]
            if mask:
                for j in np.nonzero(self.mask[b, :P] == 0)[0]:
                    self.k[b, :, j], self.v[b, :, j] = NAN, float("inf") if j % 2 else NAN
            self.k[b, :, P + n[b]:], self.v[b, :, P + n[b]:] = NAN, NAN
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.out = torch.full((N, heads * d + 16 * pad), 7.0, device="cuda").to(TYPES[self.out_type][0])

    def seen(self, b):
        n, P, a = self.n[b], self.lens[b], self.start[b]
        s = np.zeros((n, P + n), bool)
        if P:
            s[:, :P] = True if self.mask is None else self.mask[b, :P] != 0
        for i in range(n):
            at = i
            while at >= 0:
                s[i, P + at] = True
                at = self.parents[a + at]
        return torch.from_numpy(s).cuda()

    def run(self, check=True, **over):
        dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.keep = [dev(self.start), dev(self.parents), dev(np.array(self.lens, dtype=np.int32)), dev(self.mask)]
        work = torch.full((pkg.shard_tree_attention_work(self.N, self.heads, self.kv_heads, self.d),), 255, dtype=torch.uint8, device="cuda")
        self.keep.append(work)
        ptr = [x.data_ptr() if x is not None else None for x in self.keep]
        a = dict(q=self.q.data_ptr(), q_type=TYPES[self.q_type][1], k=self.k_at.data_ptr(), v=self.v_at.data_ptr(), kv_type=TYPES[self.kv_type][1],
                 out=self.out.data_ptr(), out_type=TYPES[self.out_type][1], B=self.B, N=self.N, n_heads=self.heads, n_kv_heads=self.kv_heads,
                 head_dim=self.d, capacity=self.cap, kv_strides=self.strides, tree_start=ptr[0], parents=ptr[1], lens=ptr[2], mask=ptr[3],
                 mask_stride=self.cap if self.mask is not None else 0, work=ptr[4], work_bytes=work.numel(), q_stride=self.q.stride(0),
                 out_stride=self.out.stride(0), status=self.status.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
        return pkg.shard_tree_attention(**{**a, **over}, check=check)

    def check(self, scale=None):
        G, d = self.heads // self.kv_heads, self.d
        half = lambda t: torch.finfo(TYPES[t][0]).eps / 2  # noqa: E731
        tiny = torch.finfo(TYPES[self.kv_type][0]).smallest_normal * torch.finfo(TYPES[self.kv_type][0]).eps
        scale = scale or d ** -0.5
        got = self.out[:, :self.heads * d].double().view(self.N, self.heads, d)
        worst = 0.0
        for b in range(self.B):
            n, P, a = self.n[b], self.lens[b], int(self.start[b])
            if n == 0:
                continue
            seen = self.seen(b).repeat_interleave(G, 0)
            any_ = seen.any(0)
            for h in range(self.kv_heads):
                k, v = self.k[b, h, :P + n].double(), self.v[b, h, :P + n].double()
                k, v = torch.where(any_[:, None], k, 0.0), torch.where(any_[:, None], v, 0.0)
                q = self.q[a:a + n, :self.heads * d].double().view(n, self.heads, d)[:, h * G:(h + 1) * G].reshape(n * G, d)
                p = torch.softmax((q @ k.T * scale).masked_fill(~seen, float("-inf")), 1)
                want, A = p @ v, p @ v.abs()
                S = (q.abs() @ k.abs().T * scale).masked_fill(~seen, 0).amax(1, keepdim=True)
                c = seen.sum(1, keepdim=True)
                D = (d + 2) * 2.0 ** -24 * S
                r = half(self.kv_type)
                if self.q_type == "f32":
                    D = D + r * r * S + tiny * scale * k.abs().sum(1).amax()
                    r = r * r
                tol = half(self.out_type) * want.abs() + (r + 2 * D + c.clamp(min=4) * 2.0 ** -22) * A + c * 2.0 ** -31 * v.abs().amax()
                tol = tol + (2.0 ** -25 if self.out_type == "f16" else 1e-38)
                off = (got[a:a + n, h * G:(h + 1) * G].reshape(n * G, d) - want).abs()
                assert torch.isfinite(off).all(), (b, h)
                worst = max(worst, float((off / tol).max()))
        assert worst <= 1, worst
        used = int(self.start[-1])
        assert (self.out[used:] == 7).all() and (self.out[:, self.heads * d:] == 7).all()  # what is nobody's stays
        assert self.status.item() == 0
        return worst


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q,kv", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_types_and_groups(d, q, kv, group):
    c = Case([5, 1, 9], [130, 0, 64], 2 * group, 2, d, q=q, kv=kv, holes=0.2, seed=group)
    c.run()
    c.check()


@pytest.mark.parametrize("P", [0, 1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000])
def test_cache_lengths_around_the_tiles(P):
    c = Case([1, 3, 17], [P, max(0, P - 1), P], 8, 2, 128, holes=0.1, seed=P)
    c.run()
    c.check()


@pytest.mark.parametrize("kind", ["chain", "random", "star"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 100, 255, 256])
def test_trees(kind, n):
    c = Case([n, 1, max(1, n // 2)], [77, 250, 128], 8, 2, 64, kind=kind, seed=n)
    c.run()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_large_trees_with_many_heads(d):
    c = Case([256, 0, 129, 40], [300, 10, 0, 513], 32, 2, d, q="bf16", kv="bf16", holes=0.1)
    c.run()
    c.check()


@pytest.mark.parametrize("by_entry", [False, True])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
def test_layouts_strides_and_output_types(by_entry, out):
    c = Case([6, 3], [200, 90], 12, 3, 64, q="f16", out=out, by_entry=by_entry, pad=1, holes=0.3)
    c.run()
    c.check()


def test_long_cache_is_split_and_joined():
    c = Case([4, 32, 1], [20000, 33333, 7], 8, 2, 128, holes=0.05)
    c.run()
    c.check()
    first = c.out.clone()
    c.run()
    assert torch.equal(first, c.out)  # the same bits every time


def test_many_small_requests():
    n = [(i * 7) % 5 for i in range(256)]
    c = Case(n, [(i * 13) % 200 for i in range(256)], 4, 1, 64)
    c.run()
    c.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv", ["f16", "bf16"])
def test_32_bit_queries_keep_their_precision(kv, d):
    """Relative to the result: a weight is off by 2^-21 for its exponent's 32 bits (up to 2^3), by 2^-22 each for the exponential,
    for the parts of q and of itself and for the sums of a score, at random: under 2^-19 on the whole."""
    c = Case([20, 40, 1], [500, 900, 3000], 8, 2, d, q="f32", kv=kv, holes=0.05)
    c.run()
    c.check()
    got = c.out[:, :8 * d].double().view(c.N, 8, d)
    off = whole = 0.0
    for b in range(c.B):
        n, a = c.n[b], int(c.start[b])
        end, seen = c.lens[b] + n, c.seen(b).repeat_interleave(4, 0)
        for h in range(2):
            k, v = (torch.where(seen.any(0)[:, None], x[b, h, :end].double(), 0.0) for x in (c.k, c.v))
            q = c.q[a:a + n].double().view(n, 8, d)[:, 4 * h:4 * h + 4].reshape(4 * n, d)
            want = torch.softmax((q @ k.T * d ** -0.5).masked_fill(~seen, float("-inf")), 1) @ v
            off += float((got[a:a + n, 4 * h:4 * h + 4].reshape(4 * n, d) - want).square().sum())
            whole += float(want.square().sum())
    assert off ** 0.5 <= 2.0 ** -19 * whole ** 0.5, (off / whole) ** 0.5


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q,kv", [("f32", "f16"), ("f32", "bf16"), ("f16", "f16"), ("bf16", "bf16")])
@pytest.mark.parametrize("lens", [(3, 250, 9, 100, 380, 60, 1, 130), (50, 140, 300), (100, 200)])
def test_pieces_of_one_tile_and_of_several_in_turn(q, kv, d, lens):
    """Runs of many pieces, of one tile (which one of a CTA's two streams takes alone) and of two to four, one behind the other."""
    P = [lens[b % len(lens)] for b in range(224)]
    c = Case([1 + b % 3 for b in range(224)], P, 16, 8, d, q=q, kv=kv, seed=5)
    for _ in range(5):
        c.run()
    c.check()


def exact(c, scale=None):
    """[nodes][heads][d] in 64 bits, of the nodes of requests"""
    G, d, scale = c.heads // c.kv_heads, c.d, scale or c.d ** -0.5
    out = torch.empty(c.N, c.heads, d, dtype=torch.float64, device="cuda")
    for b in range(c.B):
        n, a = c.n[b], int(c.start[b])
        if n == 0:
            continue
        end, seen = c.lens[b] + n, c.seen(b).repeat_interleave(G, 0)
        for h in range(c.kv_heads):
            k, v = (torch.where(seen.any(0)[:, None], x[b, h, :end].double(), 0.0) for x in (c.k, c.v))
            q = c.q[a:a + n, :c.heads * d].double().view(n, c.heads, d)[:, G * h:G * h + G].reshape(G * n, d)
            p = torch.softmax((q @ k.T * scale).masked_fill(~seen, float("-inf")), 1)
            out[a:a + n, G * h:G * h + G] = (p @ v).view(n, G, d)
    return out[:int(c.start[-1])]


def relative(c, want):
    """L2 distance of the outputs relative to the result, the largest over (request, head)"""
    got = c.out[:, :c.heads * c.d].double().view(c.N, c.heads, c.d)
    worst = 0.0
    for b in range(c.B):
        rows = slice(int(c.start[b]), int(c.start[b + 1]))
        if c.n[b]:
            worst = max(worst, float(((got[rows] - want[rows]).square().sum((0, 2)) / want[rows].square().sum((0, 2))).max()) ** 0.5)
    return worst


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv", ["f16", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** -140, 1e-30, 1e-6, 1e-4, 1e-3, 0.03, 100.0, 65520.0, 1e6, 1e30, 2.0 ** 125])
def test_32_bit_queries_of_any_size(kv, d, size):
    """With scale times size the same, a query of any size has the precision of one of ordinary size (bound as above)."""
    c = Case([4, 9], [300, 70], 8, 2, d, q="f32", kv=kv, holes=0.05)
    c.q = (c.q.double().clamp(-3.9, 3.9) * size).float()
    scale = float(np.float32(min(d ** -0.5 / size, 2.0 ** 120)))
    c.run(scale=scale)
    assert c.status.item() == 0
    assert relative(c, exact(c, scale)) <= 2.0 ** -19


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv", ["f16", "bf16"])
@pytest.mark.parametrize("tiles,n", [(1, 5), (2, 5), (4, 5), (16, 5), (64, 5), (3, 64), (9, 50)])
def test_32_bit_outputs_keep_their_precision_over_many_tiles(tiles, n, kv, d):
    """152 items, each of so many tiles and by one CTA where the GPU has as many SMs: the precision of one tile (bound as above)."""
    c = Case([n] * 19, [128 * tiles - n] * 19, 16, 8, d, q="f32", kv=kv, mask=False, seed=tiles, cap=128 * tiles)
    c.run()
    assert c.status.item() == 0
    assert relative(c, exact(c)) <= 2.0 ** -19


@pytest.mark.parametrize("q,kv,out", [("f16", "f16", "f16"), ("bf16", "bf16", "f32"), ("f32", "f16", "f16"), ("f32", "bf16", "bf16"), ("f32", "bf16", "f32"),
                                      ("f32", "f16", "f32")])
@pytest.mark.parametrize("n,d", [(2, 64), (2, 128), (40, 64), (20, 128)])
def test_runs_of_long_and_short_pieces(q, kv, out, n, d):
    """More items than SMs, of 133 tiles and of a few in turn, so that a CTA has several pieces, with more tiles than a stream adds up
    before it takes its sums over and with fewer.  Relative to the result: half a step each for the weights (32-bit queries: 2^-19 as
    above) and the outputs.  A tile left out or taken twice would be 2^-4."""
    B = 40
    c = Case([n, max(1, n // 2)] * (B // 2), [(17000, 300, 16800, 90, 700)[b % 5] for b in range(B)], 16, 4, d, q=q, kv=kv, out=out, holes=0.02)
    c.run()
    assert c.status.item() == 0
    half = lambda t: torch.finfo(TYPES[t][0]).eps / 2  # noqa: E731
    assert relative(c, exact(c)) <= (2.0 ** -19 if q == "f32" else half(kv)) + (0 if out == "f32" else half(out))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q,kv", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f16"), ("f32", "bf16")])
def test_every_tile_counts_once(q, kv, d):
    """Queries of zero weigh all entries alike; a value is 1 in one column, another for each tile, so that a column is the share of its
    tiles' entries that are seen: one tile more or less is a fourth of it or more.  Weights of 2^6 are exact."""
    c = Case([4, 32, 1, 40], [20000, 33333, 7, 5000], 8, 2, d, q=q, kv=kv, out="f32", holes=0.05)
    c.q.zero_()
    tile = torch.arange(c.cap, device="cuda") // 128 % d
    c.v.copy_(torch.where(torch.isfinite(c.v), torch.nn.functional.one_hot(tile, d).to(c.v.dtype), c.v))
    c.run()
    assert c.status.item() == 0
    want, got = exact(c), c.out[:int(c.start[-1])].double().view(-1, 8, d)
    assert ((got - want).abs() <= 2.0 ** -19 * want).all()


@pytest.mark.parametrize("q,kv,out", [("f16", "f16", "f32"), ("bf16", "bf16", "f32"), ("f32", "f16", "f32"), ("f32", "f16", "f16"), ("f32", "bf16", "bf16")])
@pytest.mark.parametrize("d", [64, 128])
def test_sums_over_two_thousand_tiles(q, kv, out, d):
    """All values 1, so that a result is 1 but for the sums: 1024 tiles a stream, and short pieces before them.  If the tensor unit cuts
    off an ulp a product, of a sum that grows, n products lose n * 0.72 2^-23 / 2 of it: 3.5e-4 for all of them, 4.4e-5 for the 1024
    that are added up before a sum is taken over (32-bit queries with 16-bit outputs: 1536, 6.6e-5, and the outputs' step).
    Weights of 2^18 entries are rounded at random: 2^-9 / 2^9.  152 kv heads that overlap, and so do the two requests."""
    heads, P = 152, 1 << 18
    g = torch.Generator(device="cuda").manual_seed(7)
    wide = d + 8 * heads
    k = torch.randn(P + 3, wide, generator=g, device="cuda").to(TYPES[kv][0])
    v = torch.ones_like(k)
    x = torch.randn(3, heads * d, generator=g, device="cuda").to(TYPES[q][0])
    o = torch.zeros(3, heads * d, device="cuda").to(TYPES[out][0])
    start, parents, lens, status = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, 1, 3], [-1, -1, 0], [300, P], [0]))
    work = torch.empty(pkg.shard_tree_attention_work(3, heads, heads, d), dtype=torch.uint8, device="cuda")
    pkg.shard_tree_attention(x.data_ptr(), TYPES[q][1], k.data_ptr(), v.data_ptr(), TYPES[kv][1], o.data_ptr(), TYPES[out][1], 2, 3, heads, heads, d,
                             P + 2, (8, 8, wide), start.data_ptr(), parents.data_ptr(), lens.data_ptr(), None, 0, work.data_ptr(),
                             work.numel(), status=status.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    assert status.item() == 0
    step = 0 if out == "f32" else torch.finfo(TYPES[out][0]).eps / 2
    off = (o.double() - 1).abs()
    exact_sums = q == "f32" and out == "f32"
    assert float(off[1:].mean()) <= step + (2.0 ** -19 if exact_sums else 2.0 ** -14)
    assert float(off[1:].max()) <= step + (2.0 ** -18 if exact_sums else 2.0 ** -13)
    assert float(off[0].max()) <= step + (2.0 ** -18 if q == "f32" else torch.finfo(TYPES[kv][0]).eps / 2)


@pytest.mark.parametrize("kv", ["f16", "bf16"])
def test_32_bit_queries_of_unlike_rows_and_values(kv):
    """Rows from 1e-6 to 1e6 in one batch, and a value of 1e5 among ordinary ones that K has a zero for: a part of its row is off by
    2^-38 of it at most, 2^-21 of an ordinary value."""
    c = Case([16], [333], 4, 1, 128, q="f32", kv=kv)
    c.q[:16] *= torch.logspace(-6, 6, 16, device="cuda")[:, None]
    c.run()
    c.check()
    c = Case([16], [333], 4, 1, 128, q="f32", kv=kv)
    c.q[:, ::128], c.k_at[..., 0] = 1e5, 0.0
    c.run()
    assert relative(c, exact(c)) <= 2.0 ** -19


@pytest.mark.parametrize("kv", ["f16", "bf16"])
def test_32_bit_queries_that_are_not_finite_or_zero(kv):
    c = Case([6], [200], 4, 2, 64, q="f32", kv=kv, kind="star")
    c.q[0] = 0.0
    c.q[1, 5], c.q[2, 70], c.q[3, 130] = float("inf"), NAN, -float("inf")
    c.q[4] *= 2.0 ** 120
    c.run()
    got = c.out[:6].view(6, 4, 64)
    bad = torch.zeros(6, 4, dtype=torch.bool)
    bad[1, 0] = bad[2, 1] = bad[3, 2] = True
    assert torch.equal(torch.isnan(got).all(2).cpu(), bad) and torch.equal(torch.isnan(got).any(2).cpu(), bad)
    mean = torch.stack([torch.cat([c.v[0, h, :200].double(), c.v[0, h, 200:201].double()]).mean(0) for h in (0, 0, 1, 1)])
    assert ((got[0].double() - mean).abs() <= 2.0 ** -19 * c.v[0, :, :206].double().abs().amax()).all()


@pytest.mark.parametrize("q,kv", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f16"), ("f32", "bf16")])
def test_long_cache_split_and_joined_has_the_precision_of_a_short_one(q, kv):
    """Relative to the result, per request and head: half a step each for the weights and the outputs (32-bit queries 2^-19 as above),
    however long the cache; 128 entries left out of 33333 would be 2^-4."""
    c = Case([4, 32, 1], [20000, 33333, 7], 8, 2, 128, q=q, kv=kv, holes=0.05)
    c.run()
    assert relative(c, exact(c)) <= (2.0 ** -19 if q == "f32" else torch.finfo(TYPES[kv][0]).eps)


def test_trees_that_begin_behind_other_nodes():
    """Nodes ahead of the first tree belong to nobody, whether items are cut between CTAs or not."""
    for lens in ([3000, 900], [5, 70]):
        c = Case([6, 9], lens, 8, 2, 128, extra_nodes=7)
        c.start += 4
        c.parents = np.concatenate([[-1] * 4, c.parents[:-4]]).astype(np.int32)
        c.run()
        c.check()
        assert (c.out[:4] == 7).all()


def test_no_mask_and_a_scale():
    c = Case([3, 5], [100, 129], 4, 2, 128, mask=False)
    c.run(scale=0.31)
    c.check(scale=0.31)


def test_a_cache_masked_wholly_leaves_the_tree():
    c = Case([4, 2], [300, 5], 4, 2, 64, holes=2.0)
    c.run()
    c.check()


def test_large_scores_and_weights_far_apart():
    c = Case([8], [400], 4, 1, 128)
    c.q *= 40
    c.run()
    c.check()
    c = Case([8], [400], 4, 1, 128, q="f32", kv="f16")
    c.q *= 100
    c.run()
    c.check()


@pytest.mark.parametrize("q,kv,times", [("f16", "f16", 15000.0), ("bf16", "bf16", 2.0 ** 60), ("f32", "f16", 2.0 ** 110), ("f32", "bf16", 2.0 ** 55)])
@pytest.mark.parametrize("P", [40, 300, 9000])
def test_scores_beyond_what_32_bits_resolve(q, kv, times, P):
    """Finite scores of 2^28 to 2^122: every row is its largest score's value, where the next is further below than 32 bits of the sum
    of a score's products are off (d 2^-24 of |q| |k|)."""
    c = Case([6], [P], 4, 2, 64, q=q, kv=kv)
    c.q = (c.q.float().clamp(-4, 4) * times).to(c.q.dtype)
    if kv == "f16":
        c.k.clamp_(-4, 4).mul_(4000 if q == "f16" else 1)  # NaN stays
    else:
        c.k.mul_(2.0 ** 55)
    c.run()
    assert c.status.item() == 0
    got, sure = c.out[:6].double().view(6, 2, 2, 64), 0
    assert torch.isfinite(got).all()
    for h in range(2):
        seen = c.seen(0)
        k, v = (torch.where(seen.any(0)[:, None], x[0, h, :P + 6].double(), 0.0) for x in (c.k, c.v))
        for i in range(6):
            for g in range(2):
                qq = c.q[i].double().view(2, 2, 64)[h, g]
                z, size = torch.where(seen[i], k @ qq, -torch.inf), (k.abs() @ qq.abs()).amax()
                two = z.topk(2)
                if two.values[0] - two.values[1] > 64 * 2.0 ** -23 * size:
                    sure += 1
                    assert ((got[i, h, g] - v[two.indices[0]]).abs() <= 2.0 ** -11 * v[two.indices[0]].abs() + 2.0 ** -24).all() if kv == "f16" else (
                        (got[i, h, g] - v[two.indices[0]]).abs() <= 2.0 ** -8 * v[two.indices[0]].abs()).all()
    assert sure >= 12


def test_a_nodes_infinite_values_reach_only_those_that_see_it():
    for kv in ("f16", "bf16"):
        c = Case([20, 20], [70, 128], 4, 2, 64, q=kv, kv=kv, kind="random", seed=3)
        c.run()
        clean = c.out.clone()
        node = 4
        c.k[1, :, 128 + node] = NAN
        c.v[1, :, 128 + node] = float("inf")
        c.run()
        sees = c.seen(1)[:, 128 + node].cpu().numpy()
        assert sees.any() and not sees.all()
        for i in range(20):
            same = torch.equal(c.out[i], clean[i])
            assert same, i
            row, was = c.out[20 + i], clean[20 + i]
            if sees[i]:
                assert not torch.isfinite(row[:4 * 64]).any(), i
            else:
                assert torch.equal(row, was), i


def test_infinite_value_of_a_seen_node():
    c = Case([3], [10], 2, 1, 64, kind="star")
    c.v[0, :, 11, 5] = float("inf")  # node 1's
    c.run()
    out = c.out[:3].view(3, 2, 64).float()
    assert torch.isinf(out[1, :, 5]).all() and torch.isfinite(out[1, :, 6:]).all()
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[2]).all()


def test_bad_requests_are_left_out_and_reported():
    c = Case([3, 4, 5], [40, 50, 60], 4, 2, 64)
    c.run()
    good = c.out.clone()
    for what, bit in (("negative", pkg.SHARD_TREE_LENGTH), ("capacity", pkg.SHARD_TREE_LENGTH), ("start", pkg.SHARD_TREE_START)):
        c.out.fill_(7.0)
        c.status.zero_()
        lens, start = list(c.lens), c.start.copy()
        if what == "negative":
            c.lens = [40, -1, 60]
        elif what == "capacity":
            c.lens = [40, c.cap - 3, 60]
        else:
            c.start = np.array([0, 3, 1 << 30, 12], dtype=np.int32)
        c.run()
        assert c.status.item() == bit, what
        assert torch.equal(c.out[:3], good[:3]) and (c.out[3:7] == 7).all(), what
        assert torch.equal(c.out[7:12], good[7:12]) or what == "start"
        c.lens, c.start = lens, start


def test_bad_parents_count_as_none():
    c = Case([4, 5], [40, 33], 4, 2, 64, kind="chain")
    c.parents[2], c.parents[6] = 5, -9
    c.run()
    assert c.status.item() == pkg.SHARD_TREE_PARENT
    c.status.zero_()
    c.parents[2], c.parents[6] = -1, -1
    c.check()


def test_many_more_nodes_than_the_trees_have():
    """Nodes behind the last tree count for nothing: a buffer of 2^20 of them with one small tree on a cache of 2^23 entries."""
    t = torch.Generator(device="cuda").manual_seed(1)
    N, G, d, cap = 1 << 20, 16, 64, 1 << 23
    kv = torch.empty(cap, d, dtype=torch.float16, device="cuda")
    kv[:200] = torch.randn(200, d, generator=t, device="cuda").half()
    start, parents, lens = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, 3], [-1, 0, 0], [190]))
    parents = torch.cat([parents, torch.full((N - 3,), -1, dtype=torch.int32, device="cuda")])
    q = torch.zeros(N, G * d, dtype=torch.float16, device="cuda")
    q[:3] = torch.randn(3, G * d, generator=t, device="cuda").half()
    outs = []
    for n in (3, N):
        out = torch.full((n, G * d), 7.0, dtype=torch.float16, device="cuda")
        work = torch.empty(pkg.shard_tree_attention_work(n, G, 1, d), dtype=torch.uint8, device="cuda")
        pkg.shard_tree_attention(q.data_ptr(), pkg.SHARD_F16, kv.data_ptr(), kv.data_ptr(), pkg.SHARD_F16, out.data_ptr(), pkg.SHARD_F16, 1, n, G, 1, d,
                                 cap, (cap * d, cap * d, d), start.data_ptr(), parents.data_ptr(), lens.data_ptr(), None, 0, work.data_ptr(), work.numel(),
                                 stream=torch.cuda.current_stream().cuda_stream)
        outs.append(out)
    assert torch.equal(outs[0], outs[1][:3]) and (outs[1][3:] == 7).all() and (outs[0] != 7).all()


def test_refusals():
    c = Case([2], [9], 4, 2, 64)
    E, U = pkg.SHARD_EINVAL, pkg.SHARD_EUNSUPPORTED
    for over, rc in (({"q": 0}, E), ({"work": 0}, E), ({"parents": 0}, E), ({"B": 0}, E), ({"B": 257}, E), ({"N": 0}, E), ({"capacity": 0}, E),
                     ({"n_heads": 6}, U), ({"n_kv_heads": 3}, U), ({"head_dim": 96}, U), ({"q_type": pkg.SHARD_BF16}, U), ({"kv_type": pkg.SHARD_F32}, U),
                     ({"out_type": 7}, U), ({"work_bytes": 1}, E), ({"q": c.q.data_ptr() + 2}, E), ({"kv_strides": (c.strides[0], c.strides[1], 60)}, E),
                     ({"kv_strides": (c.strides[0] + 1, c.strides[1], 64)}, E), ({"q_stride": 8}, E), ({"mask_stride": 0}, E)):
        assert c.run(check=False, **over) == rc, over
        assert pkg.shard_last_error().startswith("shard_tree_attention")
    host = torch.zeros(4096, dtype=torch.float16)
    assert c.run(check=False, q=(host.data_ptr() + 15) // 16 * 16) == E and "device memory" in pkg.shard_last_error()
    c.run()
    c.check()


def test_captured_graph_follows_the_lengths():
    c = Case([3, 7], [100, 500], 8, 2, 128, cap=2200, mask=False)
    c.run()  # loads the kernels
    torch.cuda.synchronize()
    work = torch.empty(pkg.shard_tree_attention_work(c.N, 8, 2, 128), dtype=torch.uint8, device="cuda")
    start, parents, lens, _, _ = c.keep
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.shard_tree_attention(c.q.data_ptr(), pkg.SHARD_F16, c.k_at.data_ptr(), c.v_at.data_ptr(), pkg.SHARD_F16, c.out.data_ptr(),
                                 pkg.SHARD_F16, 2, c.N, 8, 2, 128, c.cap, c.strides, start.data_ptr(), parents.data_ptr(), lens.data_ptr(), None, 0,
                                 work.data_ptr(), work.numel(), status=c.status.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    c.k_at.normal_(), c.v_at.normal_()
    for more in ([100, 500], [3, 2100], [1900, 0]):
        c.lens = more
        lens.copy_(torch.tensor(more, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        c.check()


@pytest.mark.parametrize("kv", ["f16", "bf16"])
def test_captured_graphs_of_32_bit_queries_on_two_streams(kv):
    """Sums taken over in `work`: graphs with a buffer each, replayed together with other lengths, as the eager calls."""
    s, made = torch.cuda.Stream(), []
    for seed in (1, 2):
        c = Case([5, 40], [100, 500], 8, 2, 128, q="f32", kv=kv, cap=9000, mask=False, seed=seed)
        c.k_at.normal_(), c.v_at.normal_()
        c.run()  # loads the kernels
        torch.cuda.synchronize()
        work = torch.empty(pkg.shard_tree_attention_work(c.N, 8, 2, 128), dtype=torch.uint8, device="cuda")
        start, parents, lens, _, _ = c.keep
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pkg.shard_tree_attention(c.q.data_ptr(), pkg.SHARD_F32, c.k_at.data_ptr(), c.v_at.data_ptr(), TYPES[kv][1], c.out.data_ptr(),
                                     pkg.SHARD_F32, 2, c.N, 8, 2, 128, c.cap, c.strides, start.data_ptr(), parents.data_ptr(), lens.data_ptr(), None, 0,
                                     work.data_ptr(), work.numel(), status=c.status.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
        made.append((c, graph, lens, (start, parents, work)))
    for more in ([8900, 3], [0, 8950], [4000, 5000]):
        for c, _, lens, _ in made:
            c.lens = more
            lens.copy_(torch.tensor(more, dtype=torch.int32))
        torch.cuda.synchronize()
        for _ in range(3):
            made[0][1].replay()
            with torch.cuda.stream(s):
                made[1][1].replay()
        torch.cuda.synchronize()
        for c, _, _, _ in made:
            assert c.status.item() == 0 and relative(c, exact(c)) <= 2.0 ** -19
            first = c.out.clone()
            c.run()
            assert torch.equal(first, c.out)


def test_two_streams_with_a_work_buffer_each():
    a, b = Case([9, 2], [3000, 100], 8, 2, 64, seed=1), Case([1, 30], [50, 4000], 8, 2, 64, seed=2)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(s):
            a.run()
        with torch.cuda.stream(t):
            b.run()
    torch.cuda.synchronize()
    a.check()
    b.check()


# ---------------------------------------------------------------------------
# acceptance
# ---------------------------------------------------------------------------

def plain_accept(start, parents, drafts, targets, stride, lens, mask):
    B = len(start) - 1
    path, tokens, count = np.full((B, stride), -1, np.int32), np.full((B, stride), -1, np.int32), np.zeros(B, np.int32)
    mask = mask.copy()
    for b in range(B):
        a, n = start[b], start[b + 1] - start[b]
        mask[b, lens[b]:lens[b] + n] = 0
        at = 0 if n else None
        while at is not None:
            path[b, count[b]], tokens[b, count[b]] = at, targets[a + at]
            mask[b, lens[b] + at] = 1
            count[b] += 1
            at = next((c for c in range(at + 1, n) if parents[a + c] == at and drafts[a + c] == targets[a + at]), None)
    return path, tokens, count, mask


def run_accept(start, parents, drafts, targets, stride, lens, mask, check=True):
    dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (start, parents, drafts, targets)]
    B = len(start) - 1
    path, tokens = (torch.full((B, stride), 5, dtype=torch.int32, device="cuda") for _ in range(2))
    count, status = torch.full((B,), 5, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    d_lens, d_mask = (None, None) if mask is None else (torch.from_numpy(np.asarray(lens, np.int32)).cuda(), torch.from_numpy(mask.copy()).cuda())
    pkg.shard_tree_accept(B, len(parents), *[x.data_ptr() for x in dev], stride, path.data_ptr(), tokens.data_ptr(), count.data_ptr(),
                          lens=d_lens.data_ptr() if mask is not None else None, attention_mask=d_mask.data_ptr() if mask is not None else None,
                          mask_stride=0 if mask is None else mask.shape[1], status=status.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    return path.cpu().numpy(), tokens.cpu().numpy(), count.cpu().numpy(), None if mask is None else d_mask.cpu().numpy(), status.item()


@pytest.mark.parametrize("kind", ["chain", "random", "star"])
@pytest.mark.parametrize("n", [[1], [2, 0, 3], [256, 1, 255, 33], [64] * 70])
@pytest.mark.parametrize("tokens", [1, 2, 40])
def test_accept(kind, n, tokens):
    g = np.random.default_rng(sum(n) + tokens)
    start = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    parents = np.array(trees(n, kind, g) + [0], dtype=np.int32)
    drafts, targets = (g.integers(0, tokens, len(parents)).astype(np.int32) for _ in range(2))
    lens = g.integers(0, 100, len(n))
    mask = g.integers(0, 2, (len(n), 400)).astype(np.uint8)
    want = plain_accept(start, parents, drafts, targets, max(n) + 3, lens, mask)
    got = run_accept(start, parents, drafts, targets, max(n) + 3, lens, mask)
    for w, x in zip(want, got):
        assert np.array_equal(w, x)
    assert got[4] == 0
    bare = run_accept(start, parents, drafts, targets, max(n) + 3, None, None)
    assert all(np.array_equal(w, x) for w, x in zip(want[:3], bare[:3]))


def test_accept_leaves_out_what_is_wrong():
    start, parents = np.array([0, 3, 6, 9], np.int32), np.array([-1, 0, 1, -1, 0, 1, -1, 0, 7], np.int32)
    drafts, targets, mask = np.zeros(9, np.int32), np.zeros(9, np.int32), np.full((3, 20), 9, np.uint8)
    path, tokens, count, after, status = run_accept(start, parents, drafts, targets, 3, [0, 18, 4], mask)
    assert status == pkg.SHARD_TREE_LENGTH | pkg.SHARD_TREE_PARENT
    assert count.tolist() == [3, 0, 2] and path.tolist() == [[0, 1, 2], [5, 5, 5], [0, 1, -1]]
    assert (after[1] == 9).all() and after[2].tolist() == [9] * 4 + [1, 1, 0] + [9] * 13
    path, _, count, _, status = run_accept(start, parents, drafts, targets, 2, None, None)
    assert status == pkg.SHARD_TREE_START and count.tolist() == [0, 0, 0] and (path == 5).all()
    _, _, count, _, status = run_accept(np.array([0, 3, 1 << 30, 9], np.int32), parents, drafts, targets, 3, None, None)
    assert status == pkg.SHARD_TREE_START and count.tolist() == [3, 0, 0]


def test_accept_keeps_node_0_whatever_its_parent():
    start, zero = np.array([0, 3], np.int32), np.zeros(3, np.int32)
    for first in (-1, 0, 2, -7):
        path, _, count, _, status = run_accept(start, np.array([first, 0, 1], np.int32), zero, zero, 3, None, None)
        assert path.tolist() == [[0, 1, 2]] and count.tolist() == [3] and status == (0 if first == -1 else pkg.SHARD_TREE_PARENT)


def test_accept_refusals():
    x = torch.zeros(16, dtype=torch.int32, device="cuda").data_ptr()
    def rc(*a, **k):
        return pkg.shard_tree_accept(*a, **k, check=False)
    E = pkg.SHARD_EINVAL
    assert rc(0, 4, x, x, x, x, 4, x, x, x) == E and rc(257, 4, x, x, x, x, 4, x, x, x) == E and rc(1, 0, x, x, x, x, 4, x, x, x) == E
    assert rc(1, 4, 0, x, x, x, 4, x, x, x) == E and rc(1, 4, x, x, x, x, 0, x, x, x) == E and rc(1, 4, x, x, x, x, 4, x, x, 0) == E
    assert rc(1, 4, x, x, x, x, 4, x, x, x, lens=x) == E and rc(1, 4, x, x, x, x, 4, x, x, x, lens=x, attention_mask=x, mask_stride=0) == E
