"""The cache operators against their definitions in 64 bits (include/spechub_cache.h).

Tolerances.  u = finfo(type).eps / 2 is the relative error of one rounding.
  append     the rotated value x0 cos - x1 sin is rounded once: u |r| (or half the smallest number's spacing); before that,
             cos and sin carry the rounding of the angle's fraction of a turn (2^-25 pi) and 2 ulp of the function, products and
             sum one rounding each: below 6e-7 (|x0| + |x1|) together.
  attention  out is rounded once: u |out|.  Every weight is rounded once for its product: u sum p |v|, and in fp16, where small
             weights lie among the subnormals, 2^-25 of the weight 1 per key.  A score is a sum of D products in 32 bits, each
             addition off by at most 2^-23 of the sum of magnitudes (a factor of two for an adder that cuts off), which is off in
             the exponent by delta = D 2^-23 scale sum |q k|; the exponential's argument and result add 2^-21 (1 + |s - max|).  The
             sums over n keys are off by at most n 2^-23 in relation.  lse is off by the same without the two u.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def sh():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2411_05289_b200 as lib

    lib.load_library()
    return lib


def make_cache(gen, pages, ps, hk, d, dt, layout="nhd", layers=None, fill=None):
    shape = (pages, hk, ps, d) if layout == "hnd" else (pages, ps, hk, d)
    if layers is not None:
        shape = (layers,) + shape
    if layout == "pair":     # keys and values side by side in one tensor, with a gap behind every head
        t = torch.randn(shape[:-1] + (2 * d + 8,), generator=gen, device="cuda")
        t = (t if fill is None else torch.full_like(t, fill)).to(dt)
        return t[..., :d], t[..., d:2 * d]
    out = []
    for _ in range(2):
        t = torch.randn(shape, generator=gen, device="cuda") if fill is None else torch.full(shape, fill, device="cuda")
        t = t.to(dt)
        out.append(t.transpose(-3, -2) if layout == "hnd" else t)
    return out


class Case:
    """A batch over a paged cache; what no sequence uses is NaN."""

    def __init__(self, seed, lens, nodes, hk, g, d, ps, dt="bf16", layout="nhd", shared=0, mask=None, q_sd=1.5, strided_q=False, spare=3):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        self.lens_list, self.n, self.hk, self.g, self.d, self.ps, self.dt = list(lens), nodes, hk, g, d, ps, TYPES[dt]
        b = len(self.lens_list)
        need = [max(0, -(-(x + nodes) // ps)) if x >= 0 else 0 for x in self.lens_list]
        self.shared = shared
        ns = -(-shared // ps)
        total = sum(need) + ns + spare
        ids = self.rng.permutation(total).astype(np.int32)
        width = max(max(need), 1)
        table = np.full((b, width), 123456789, np.int32)   # what is not in use is no page
        at = ns
        for i, c in enumerate(need):
            table[i, :c] = ids[at:at + c]
            at += c
        self.shared_pages = torch.from_numpy(ids[:ns].copy()).cuda()
        self.pages = torch.from_numpy(table).cuda()
        self.lens = torch.tensor(self.lens_list, dtype=torch.int32, device="cuda")
        self.kc, self.vc = make_cache(self.gen, total, ps, hk, d, self.dt, layout, fill=math.nan)
        self.table, self.ids_shared = table, ids[:ns]
        for i, x in enumerate(self.lens_list):
            if x >= 0:
                self.put(table[i], x + nodes)
        self.put(ids[:ns], shared)
        q = torch.randn((b, nodes, hk * g + (2 if strided_q else 0), d), generator=self.gen, device="cuda") * q_sd
        self.q = q.to(self.dt)[:, :, : hk * g]
        sees = np.tril(np.ones((nodes, nodes), bool)) if mask is None else mask
        self.sees = sees
        self.mask = torch.from_numpy(pack(sees)).cuda()

    def put(self, pages, count):
        """Ordinary values for the first `count` slots of these pages."""
        for at in range(0, count, self.ps):
            m = min(self.ps, count - at)
            for c in (self.kc, self.vc):
                c[int(pages[at // self.ps]), :m] = torch.randn((m, self.hk, self.d), generator=self.gen, device="cuda").to(self.dt)

    def run(self, sh, **kw):
        if self.shared:
            kw.update(shared_pages=self.shared_pages, shared_len=self.shared)
        return sh.spechub_tree_attention(self.q, self.kc, self.vc, self.pages, self.lens, self.mask, **kw)

    def flat(self, cache, pages, count):
        idx = torch.from_numpy(np.asarray(pages[: -(-count // self.ps)], np.int64)).cuda()
        return cache[idx].flatten(0, 1)[:count].double()

    def check(self, got, scale=None, skip=()):
        scale = self.d ** -0.5 if scale is None else scale
        u = torch.finfo(self.dt).eps / 2
        tiny = 2.0 ** -25 if self.dt == torch.float16 else 0.0
        for i, x in enumerate(self.lens_list):
            if x < 0 or i in skip:
                continue
            sees = torch.from_numpy(self.sees if self.sees.ndim == 2 else self.sees[i]).cuda()
            k = torch.cat((self.flat(self.kc, self.ids_shared, self.shared), self.flat(self.kc, self.table[i], x + self.n)))
            v = torch.cat((self.flat(self.vc, self.ids_shared, self.shared), self.flat(self.vc, self.table[i], x + self.n)))
            k, v = k.permute(1, 2, 0), v.transpose(0, 1)                                   # Hk, D, L and Hk, L, D
            q = self.q[i].double().reshape(self.n, self.hk, self.g, self.d).permute(1, 2, 0, 3).reshape(self.hk, self.g * self.n, self.d)
            vis = torch.ones((self.n, self.shared + x + self.n), dtype=torch.bool, device="cuda")
            vis[:, self.shared + x:] = sees
            vis = vis.repeat(self.g, 1)
            s = torch.where(vis, (q @ k) * scale, -math.inf)
            size = torch.where(vis, (q.abs() @ k.abs()) * scale, 0.0).amax(-1)
            top = s.amax(-1)
            ref = torch.where(top == -math.inf, 0.0, top)
            p = torch.exp(s - ref[..., None])
            total = p.sum(-1)
            some = total > 0
            w = torch.where(some[..., None], p / total[..., None], 0.0)
            seen_v = torch.where(vis.any(0)[:, None], v, 0.0)
            o, mag = w @ seen_v, w @ seen_v.abs()
            count = s.shape[-1]
            delta = self.d * 2.0 ** -23 * size + 2.0 ** -21 * (1 + size) + count * 2.0 ** -23
            tol = u * o.abs() + (u + 4 * delta[..., None]) * 1.01 * mag + count * tiny * seen_v.abs().amax(1, keepdim=True) + 1e-30
            tol = tol + (2.0 ** -25 if self.dt == torch.float16 else 0.0)
            back = lambda t, *e: t.reshape(self.hk, self.g, self.n, *e).permute(2, 0, 1, *range(3, 3 + len(e))).reshape(self.n, self.hk * self.g, *e)  # noqa: E731
            far = (got["out"][i].double() - back(o, self.d)).abs()
            assert bool((far <= back(tol, self.d)).all()), (i, x, float((far / back(tol, self.d)).nan_to_num(math.inf).amax()))
            lse = torch.where(some, ref + torch.log(total), -math.inf)
            far = (got["lse"][i].double() - back(lse)).abs()
            ok = (far <= back(2 * delta + 2.0 ** -22 * lse.abs())) | (got["lse"][i].double() == back(lse))
            assert bool(ok.all()), (i, x, "lse", float(far.nan_to_num(math.inf).amax()))


def pack(sees):
    n = sees.shape[-1]
    bits = np.zeros(sees.shape[:-1] + (32 * -(-n // 32),), np.uint8)
    bits[..., :n] = sees
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32)


def tree_mask(n, k=2):
    sees = np.eye(n, dtype=bool)
    for i in range(1, n):
        sees[i] |= sees[(i - 1) // k]
    return sees


# ---- append ---------------------------------------------------------------------------------------------------

def rotate64(x, pos, freq, interleaved):
    """In 64 bits, and the magnitudes that its error goes by."""
    r = 2 * len(freq)
    i = torch.arange(r // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    ang = (pos[..., None] * freq)[..., None, :]
    y, m = x.clone(), torch.zeros_like(x)
    y[..., a] = x[..., a] * ang.cos() - x[..., b] * ang.sin()
    y[..., b] = x[..., a] * ang.sin() + x[..., b] * ang.cos()
    m[..., a] = m[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, m


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("lens,n,hk,g,d,rotated,ps,layout,offset", [
    ([0], 1, 1, 1, 64, 64, 8, "nhd", 0),
    ([17], 7, 8, 4, 128, 128, 16, "nhd", 0),
    ([5, 0, 31, -1, 64], 5, 2, 3, 64, 32, 32, "hnd", 1000003),
    ([100, 3], 33, 3, 1, 128, 16, 64, "pair", 7),
    ([9, 1], 300, 1, 2, 64, 0, 128, "nhd", 2),
    ([1023, 1024, 1025], 2, 2, 7, 128, 112, 1024, "hnd", 123456789),
])
def test_append(sh, dt, interleaved, lens, n, hk, g, d, rotated, ps, layout, offset):
    c = Case(1, lens, n, hk, g, d, ps, dt, layout, strided_q=True)
    b, u = len(lens), torch.finfo(c.dt).eps / 2
    small = 2.0 ** -25 if dt == "fp16" else 0.0
    packed = torch.randn((b, n, 2 * hk, d), generator=c.gen, device="cuda").to(c.dt)   # as a projection leaves them
    k, v = packed[:, :, :hk], packed[:, :, hk:]
    freq = (10000.0 ** (-torch.arange(0, rotated, 2, dtype=torch.float64) / max(1, rotated))).float().cuda()
    depth = torch.from_numpy(tree_mask(n).sum(1).astype(np.int32) - 1).cuda()
    before = [x.clone() for x in (c.kc, c.vc)]
    q_out = torch.full((b, n, hk * g, d), 7.0, dtype=c.dt, device="cuda")
    got = sh.spechub_cache_append(c.q, k, v, c.kc, c.vc, c.pages, c.lens, depth, freq if rotated else None, offset, interleaved, q_out=q_out)
    assert got["q"].data_ptr() == q_out.data_ptr() and got["status"].tolist() == [0] * b
    for i, x in enumerate(lens):
        if x < 0:
            assert bool((q_out[i] == 7.0).all())
            continue
        pos = (offset + x + depth).double()
        for src, dst in ((c.q[i], got["q"][i]), (k[i], None), (v[i], None)):
            is_v = src.data_ptr() == v[i].data_ptr()
            if dst is None:
                cache, old = (c.vc, before[1]) if is_v else (c.kc, before[0])
                slots = [(int(c.table[i][(x + m) // ps]), (x + m) % ps) for m in range(n)]
                dst = torch.stack([cache[p, o] for p, o in slots])
                for p, o in slots:      # what is left must be what was there
                    old[p, o] = cache[p, o]
            if is_v:
                assert torch.equal(dst, src)
                continue
            want, mag = rotate64(src.double(), pos, freq.double(), interleaved)
            assert bool(((dst.double() - want).abs() <= u * want.abs() * (1 + 1e-6) + 6e-7 * mag + small).all())
            assert torch.equal(dst[..., rotated:], src[..., rotated:])
    for new, old in zip((c.kc, c.vc), before):
        assert torch.equal(new.nan_to_num(-99.0), old.nan_to_num(-99.0))


def test_append_in_place_and_without_queries_and_with_a_tree_per_sequence(sh):
    c = Case(2, [10, 20], 4, 2, 2, 64, 16)
    k, v = (torch.randn((2, 4, 2, 64), generator=c.gen, device="cuda").to(c.dt) for _ in range(2))
    freq = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).float().cuda()
    depth = torch.tensor([[0, 1, 1, 2], [0, 1, 2, 3]], dtype=torch.int32, device="cuda")
    want = sh.spechub_cache_append(c.q, k, v, c.kc, c.vc, c.pages, c.lens, depth, freq)["q"].clone()
    kept = [x.clone() for x in (c.kc, c.vc)]
    # sequence 1 is a chain: the same as no table
    alone = sh.spechub_cache_append(c.q[1:], k[1:], v[1:], c.kc, c.vc, c.pages[1:], c.lens[1:], None, freq)["q"]
    assert torch.equal(alone[0], want[1])
    got = sh.spechub_cache_append(None, k, v, c.kc, c.vc, c.pages, c.lens, depth, freq)
    assert set(got) == {"status"}
    for new, old in zip((c.kc, c.vc), kept):
        assert torch.equal(new.nan_to_num(-99.0), old.nan_to_num(-99.0))
    q = c.q.clone()
    assert sh.spechub_cache_append(q, k, v, c.kc, c.vc, c.pages, c.lens, depth, freq, q_out=q)["q"].data_ptr() == q.data_ptr()
    assert torch.equal(q, want)


def test_append_leaves_bad_pages_out(sh):
    c = Case(3, [14, 14, 14], 4, 2, 1, 64, 8)     # slots 14..17: pages 1 and 2 of each row
    k, v = (torch.randn((3, 4, 2, 64), generator=c.gen, device="cuda").to(c.dt) for _ in range(2))
    bad = c.pages.clone()
    bad[0, 1], bad[1, 2] = -1, c.kc.shape[0]
    before = [x.clone() for x in (c.kc, c.vc)]
    got = sh.spechub_cache_append(None, k, v, c.kc, c.vc, bad, c.lens)
    assert got["status"].tolist() == [128, 128, 0]
    for new, old, x in ((c.kc, before[0], k), (c.vc, before[1], v)):
        for i, slots in enumerate(([16, 17], [14, 15], [14, 15, 16, 17])):
            for s in slots:
                old[int(c.table[i][s // 8]), s % 8] = x[i, s - 14]
        assert torch.equal(new.nan_to_num(-99.0), old.nan_to_num(-99.0))
    short = sh.spechub_cache_append(None, k, v, c.kc, c.vc, c.pages[:, :2].contiguous(), c.lens)   # the table ends at slot 16
    assert short["status"].tolist() == [128] * 3


# ---- attention ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("lens,n,hk,g,d,ps,layout,shared", [
    ([0], 1, 1, 1, 64, 8, "nhd", 0),                       # one token, nothing before it
    ([1], 1, 2, 4, 128, 16, "nhd", 0),
    ([126, 127, 128, 129], 1, 2, 4, 128, 16, "hnd", 0),    # tiles of keys end at the context's end, or at the node's
    ([1500], 7, 8, 4, 128, 16, "nhd", 0),
    ([0, 5, 250, 700], 31, 2, 4, 128, 64, "nhd", 0),
    ([97, 98, 225], 31, 1, 3, 64, 32, "hnd", 0),
    ([40, 300, -1, 12], 13, 2, 5, 64, 8, "pair", 0),
    ([64, 2000], 1, 1, 16, 64, 128, "nhd", 0),
    ([1000, 20], 33, 1, 8, 128, 256, "hnd", 0),            # more rows than one tile holds
    ([3], 130, 2, 1, 128, 16, "nhd", 0),                   # a tree of five words
    ([513], 300, 1, 2, 64, 1024, "nhd", 0),
    ([0], 1, 1, 1, 64, 8, "nhd", 1),                       # a prefix in common
    ([10, 0, 129], 7, 2, 4, 128, 16, "nhd", 128),
    ([100] * 9, 31, 1, 4, 128, 64, "hnd", 1000),
    ([5, -1, 600, -1], 3, 2, 7, 64, 32, "nhd", 333),
    ([0] * 200, 1, 2, 1, 64, 8, "nhd", 65),
    ([70, 300], 5, 2, 33, 128, 16, "nhd", 0),              # tiles of 99 rows
    ([600], 2, 1, 128, 64, 32, "hnd", 0),
])
def test_attention(sh, dt, lens, n, hk, g, d, ps, layout, shared):
    c = Case(10 + n, lens, n, hk, g, d, ps, dt, layout, shared, tree_mask(n), strided_q=True)
    got = c.run(sh)
    assert got["status"].tolist() == [0] * len(lens)
    c.check(got)


@pytest.mark.parametrize("seed", range(6))
def test_drawn_batches(sh, seed):
    """Lengths, trees, heads, pages and prefixes as they come."""
    r = np.random.default_rng(1000 + seed)
    for _ in range(6):
        n = int(r.choice([1, 1, 2, 5, 17, 31, 64, 70, 129]))
        g, hk, d = int(r.choice([1, 2, 3, 4, 5, 8, 16])), int(r.choice([1, 2, 3])), int(r.choice([64, 128]))
        lens = [int(x) if r.random() > 0.1 else -1 for x in r.integers(0, r.choice([2, 140, 1500]), r.integers(1, 12))]
        shared = int(r.choice([0, 0, 1, 127, 128, 129, 900]))
        ps, layout = int(r.choice([8, 16, 32, 64, 128, 256])), str(r.choice(["nhd", "hnd", "pair"]))
        c = Case(int(r.integers(1 << 30)), lens, n, hk, g, d, ps, str(r.choice(["bf16", "fp16"])), layout, shared,
                 tree_mask(n, int(r.choice([1, 2, 3]))), strided_q=bool(r.random() < 0.5))
        got = c.run(sh)
        assert got["status"].tolist() == [0] * len(lens)
        c.check(got)


@pytest.mark.parametrize("lens,n,hk,g,d,shared", [
    ([40, 7, 300, 0, 12], 7, 2, 4, 128, 300),       # four sequences' rows in a tile
    ([5, 60, 2], 31, 1, 4, 64, 129),                # one
    ([5, -1, 200], 40, 1, 7, 128, 700),             # a sequence's rows in several tiles
    ([1, 2, 3] * 30, 1, 1, 8, 64, 1000),
    ([50, 9], 3, 1, 128, 64, 64),                   # a node's heads are a tile
])
def test_queries_with_gaps_between_sequences(sh, lens, n, hk, g, d, shared):
    """... and between nodes and heads: sequences do not follow each other as their nodes do."""
    c = Case(50, lens, n, hk, g, d, 16, "bf16", "nhd", shared, tree_mask(n))
    packed = c.run(sh)
    c.check(packed)
    wide = torch.full((len(lens) + 1, n + 2, hk * g + 3, d + 8), math.nan, dtype=c.dt, device="cuda")
    wide[1:, 1:-1, 2:-1, :d] = c.q
    c.q = wide[1:, 1:-1, 2:-1, :d]
    got = c.run(sh)
    c.check(got)
    room = torch.full_like(wide, 3.0)
    view = room[1:, 1:-1, 2:-1, :d]
    c.run(sh, out=dict(out=view, lse=torch.empty_like(got["lse"]), status=torch.empty_like(got["status"])))
    for i, x in enumerate(lens):
        assert torch.equal(view[i], got["out"][i] if x >= 0 else torch.full_like(view[i], 3.0))
    view.fill_(3.0)
    assert bool((room == 3.0).all())    # nothing is written beside the rows


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_peaked_and_flat_scores(sh, dt, d):
    for q_sd, scale in ((0.0, None), (30.0, None), (1.0, 1e-6), (2.0, 1.0)):
        c = Case(5, [700, 64], 6, 2, 4, d, 32, dt, "nhd", 150, tree_mask(6), q_sd=q_sd)
        c.check(c.run(sh, scale=scale), scale)


def test_scores_that_grow_along_the_keys(sh):
    """The running maximum rises in every tile: what was summed has to follow it."""
    c = Case(6, [1100], 3, 1, 4, 128, 64, "bf16", "hnd", 400, tree_mask(3))
    ramp = lambda m: (torch.arange(m, device="cuda")[:, None] * 0.02).expand(m, 128)  # noqa: E731
    c.q.copy_(torch.rand(c.q.shape, generator=c.gen, device="cuda") * 0.5)
    for pages, count in ((c.ids_shared, c.shared), (c.table[0], 1103)):
        for at in range(0, count, 64):
            m = min(64, count - at)
            c.kc[int(pages[at // 64]), :m, 0] = (ramp(at + m)[at:] + torch.randn((m, 128), generator=c.gen, device="cuda")).to(c.dt)
    c.check(c.run(sh))


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d,lens,n,g,shared", [(64, [700, 0, 130], 7, 4, 0), (128, [700, 0, 130], 40, 4, 300), (128, [500], 1, 1, 0), (64, [390], 62, 4, 0)])
def test_scores_that_jump_within_a_tile(sh, dt, d, lens, n, g, shared):
    """By 2^10 to 2^100 and back, at places inside tiles and their parts, for some of the rows of a warp only."""
    c = Case(33, lens, n, 2, g, d, 16, dt, "nhd", shared)
    u = torch.nn.functional.normalize(torch.randn(d, generator=c.gen, device="cuda"), dim=0)
    c.q += ((2.0 * d ** 0.5) * u).to(c.dt)
    c.q[:, ::3] -= ((2.0 * d ** 0.5) * u).to(c.dt)      # (these see no jumps)
    jumps = ((40, 5.0), (64, 12.0), (70, -9.0), (100, 20.0), (128, 8.0), (190, 30.0), (193, -30.0), (260, 35.0), (383, 33.0), (385, 12.0), (450, 20.0), (640, 30.0))
    for ids, count in [(c.ids_shared, shared)] + [(c.table[i], x + n) for i, x in enumerate(lens)]:
        for at, by in jumps:
            if at < count:
                page = c.kc[int(ids[at // 16])]
                page[at % 16] += (by * u).to(c.dt)
    got = c.run(sh)
    assert not got["status"].any()
    c.check(got)


def test_masks_of_any_kind(sh):
    """Rows that see no node, only others, or all; one mask per sequence; a context of nothing leaves such rows empty."""
    rng = np.random.default_rng(3)
    masks = rng.random((4, 40, 40)) < np.array([0.0, 0.1, 0.5, 1.0])[:, None, None]
    masks[1, 7] = False
    c = Case(7, [0, 0, 100, 31], 40, 2, 2, 64, 16, "bf16", "nhd", 0, masks)
    got = c.run(sh)
    c.check(got)
    assert bool((got["out"][0] == 0).all()) and bool((got["lse"][0] == -math.inf).all())
    assert bool((got["out"][1, 7] == 0).all()) and bool((got["lse"][1, 7] == -math.inf).all())


def test_values_that_are_no_numbers_concern_the_rows_that_see_them(sh):
    """NaN and infinities in the keys and values of one branch of the tree: rows of other branches are what they were."""
    n, sees = 31, tree_mask(31)
    c = Case(8, [97, 200, 1], n, 2, 4, 128, 16, "bf16", "nhd", 130, sees)
    clean = c.run(sh)
    c.check(clean)
    for bad in (math.nan, math.inf, -math.inf):
        for node in (1, 30):
            for cache in (c.kc, c.vc):
                kept = cache.clone()
                for i, x in enumerate(c.lens_list):
                    cache[int(c.table[i][(x + node) // 16]), (x + node) % 16, 1, 5] = bad
                got = c.run(sh)
                hit = torch.from_numpy(sees[:, node]).cuda()
                for key in ("out", "lse"):
                    assert torch.equal(got[key][:, ~hit], clean[key][:, ~hit])
                    assert torch.equal(got[key][:, :, :4], clean[key][:, :, :4])
                if cache is c.vc:
                    seen = got["out"][:, hit][:, :, 4:, 5].float()
                    assert bool(seen.isnan().all() if math.isnan(bad) else (seen == bad).all())
                    assert torch.equal(got["lse"], clean["lse"])
                elif math.isnan(bad):
                    assert bool(got["out"][:, hit][:, :, 4:].isnan().all())
                cache.copy_(kept)


def test_absent_sequences_are_left_as_they_were(sh):
    c = Case(9, [50, -1, 300, -5], 4, 2, 2, 64, 16, shared=40)
    out = c.run(sh)
    for t in out.values():
        t.fill_(5)
    got = c.run(sh, out=out)
    assert got["out"].data_ptr() == out["out"].data_ptr()
    for i in (1, 3):
        assert bool((got["out"][i] == 5).all()) and bool((got["lse"][i] == 5).all())
    assert got["status"].tolist() == [0] * 4
    c.check(got)


def test_bad_pages_read_as_zeros(sh):
    c = Case(11, [100, 100, 100], 5, 1, 4, 64, 32, shared=64)
    good = c.run(sh)
    bad = c.pages.clone()
    bad[0, 1], bad[2, 0] = c.kc.shape[0], -7
    got = sh.spechub_tree_attention(c.q, c.kc, c.vc, bad, c.lens, c.mask, shared_pages=c.shared_pages, shared_len=64)
    assert got["status"].tolist() == [128, 0, 128]
    for key in ("out", "lse"):
        assert torch.equal(got[key][1], good[key][1])
    for cache in (c.kc, c.vc):
        cache[int(c.table[0][1])] = 0
        cache[int(c.table[2][0])] = 0
    c.check(got)
    # a shared page that is none concerns everybody; behind the table's end there is nothing
    shared = torch.tensor([int(c.ids_shared[0]), -1], dtype=torch.int32, device="cuda")
    assert sh.spechub_tree_attention(c.q, c.kc, c.vc, c.pages, c.lens, c.mask, shared_pages=shared, shared_len=64)["status"].tolist() == [128] * 3
    assert sh.spechub_tree_attention(c.q, c.kc, c.vc, c.pages, c.lens, c.mask, shared_pages=shared, shared_len=32)["status"].tolist() == [0] * 3
    cut = sh.spechub_tree_attention(c.q, c.kc, c.vc, c.pages[:, :2].contiguous(), c.lens, c.mask)
    assert cut["status"].tolist() == [128] * 3
    d = Case(11, [64], 1, 1, 4, 64, 32)
    d.kc, d.vc, d.q, d.table = c.kc, c.vc, c.q[1:2, :1], c.table[1:2]
    mine = torch.zeros((1, 1), dtype=torch.int32, device="cuda")   # (a node that sees nothing)
    two = torch.tensor([64], dtype=torch.int32, device="cuda")
    want = sh.spechub_tree_attention(d.q, d.kc, d.vc, c.pages[1:2], two, mine)
    torch.testing.assert_close(cut["lse"][1, 0], want["lse"][0, 0], rtol=1e-6, atol=1e-6)


def test_an_enormous_length_ends_at_the_table(sh):
    c = Case(12, [40], 2, 1, 1, 64, 8)
    far = torch.tensor([2147483647], dtype=torch.int32, device="cuda")
    got = sh.spechub_tree_attention(c.q, c.kc, c.vc, c.pages, far, c.mask)
    assert got["status"].tolist() == [128]
    assert sh.spechub_cache_append(None, c.q, c.q, c.kc, c.vc, c.pages, far)["status"].tolist() == [128]


def test_offsets_beyond_32_bits(sh):
    """A cache of more than 2^32 elements: pages at its far end."""
    pages, ps, hk, d = 2200, 256, 64, 128
    cache = torch.empty((pages, ps, hk, d), dtype=torch.bfloat16, device="cuda")
    assert cache.numel() > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.tensor([[pages - 1, 3, pages - 2]], dtype=torch.int32, device="cuda")
    for p in table[0].tolist():
        cache[p].normal_(generator=gen)
    q = torch.randn((1, 5, hk, d), generator=gen, device="cuda").bfloat16()
    k = torch.randn((1, 5, hk, d), generator=gen, device="cuda").bfloat16()
    lens = torch.tensor([600], dtype=torch.int32, device="cuda")
    sh.spechub_cache_append(None, k, k, cache, cache, table, lens)
    assert torch.equal(cache[pages - 2, 88:93], k[0])
    near = cache[table[0].long()].clone()
    mask = torch.from_numpy(pack(tree_mask(5))).cuda()
    got = sh.spechub_tree_attention(q, cache, cache, table, lens, mask)
    want = sh.spechub_tree_attention(q, near, near, torch.arange(3, dtype=torch.int32, device="cuda")[None], lens, mask)
    for key in got:
        assert torch.equal(got[key], want[key])
    path = torch.tensor([[0, 2, 4]], dtype=torch.int32, device="cuda")
    assert sh.spechub_cache_accept(cache, cache.clone(), table, lens, path, 5)["lens"].tolist() == [603]
    assert torch.equal(cache[pages - 2, 88:91], k[0, [0, 2, 4]])


def test_workspace_stays_small_without_a_prefix(sh):
    """Two pieces per SM at most, whatever the batch: not one for every block."""
    import ctypes

    from test_cache_refusals import Desc

    lib = sh.load_library()
    lib.spechub_tree_attention_workspace_bytes.restype = ctypes.c_size_t
    size = {}
    for batch in (64, 4096):
        d = Desc(ctypes.sizeof(Desc), 1, 1, batch, 31, 32, 8, 128, 16, 10, 1, 100, 100, 4096, 4096)
        size[batch] = lib.spechub_tree_attention_workspace_bytes(ctypes.byref(d), ctypes.c_int64(0))
    assert size[4096] < size[64] + 4 * 5000 < 32 << 20


def test_results_repeat(sh):
    c = Case(13, [900, 0, 333, 128, 5000], 7, 2, 4, 128, 16, shared=200)
    first = c.run(sh)
    for _ in range(3):
        again = c.run(sh)
        for key in first:
            assert torch.equal(first[key], again[key])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,n,g,shared", [
    ([0] * 13, 31, 32, 5000),        # a block of one tile of rows, then blocks of two with a tile of keys each
    ([0, 1, 200, 0] * 9, 13, 32, 130),
    ([0, 300, 1, 0, 129] * 9, 5, 32, 0),
    ([0, 1] * 100, 1, 8, 0),         # all of one tile
])
def test_short_pieces_one_after_the_other(sh, d, lens, n, g, shared):
    """Pieces of a single tile of keys, which the parts of a block pass at different times."""
    case = Case(77, lens, n, 1, g, d, 16, shared=shared)
    first = {k: v.clone() for k, v in case.run(sh).items()}
    assert not first["status"].any()
    case.check(first)
    for _ in range(50):
        again = case.run(sh)
        assert not again["status"].any()
        assert torch.equal(again["out"], first["out"]) and torch.equal(again["lse"], first["lse"])


def test_other_streams_and_captured_calls(sh):
    """A captured call is replayed with other lengths, tables and queries; two graphs on two streams do not share anything."""
    c = Case(14, [400, 50, 1], 7, 2, 4, 64, 16, shared=100, mask=tree_mask(7))
    other = Case(15, [30, 700, 2], 7, 2, 4, 64, 16, shared=100, mask=tree_mask(7))
    want, want2 = c.run(sh), other.run(sh)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(sh, stream=side)
    torch.cuda.synchronize()
    for key in want:
        assert torch.equal(got[key], want[key])
    graphs, outs = [], []
    for x in (c, other):
        x.run(sh)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(x.run(sh))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, (want, want2)):
        for key in w:
            assert torch.equal(o[key], w[key])
    c.lens.copy_(torch.tensor([17, 50, -1], dtype=torch.int32))
    graphs[0].replay()
    torch.cuda.synchronize()
    c.lens_list = [17, 50, -1]
    c.check(outs[0])


# ---- accept ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("layout,ps,d,layers", [("nhd", 8, 64, 3), ("hnd", 16, 128, 2), ("pair", 32, 64, None), ("nhd", 1024, 128, 1)])
def test_accept(sh, dt, layout, ps, d, layers):
    gen, rng = torch.Generator(device="cuda").manual_seed(4), np.random.default_rng(4)
    lens, n = [0, 7, 1020, -1, 13, 30, 8], 31
    paths = [[0, 2, 6, 14, 30], [0, 1, 3, 7, 15], [0, 2, 5, -1, -1], [0, 1, -1, -1, -1], [0, -1, -1, -1, -1], [0, 1, 4, 9, 20],
             [-1, -1, -1, -1, -1]]
    need = [-(-(max(0, x) + n) // ps) for x in lens]
    ids = rng.permutation(sum(need) + 2).astype(np.int32)
    table = np.full((len(lens), max(need)), -1, np.int32)
    for i, c in enumerate(need):
        table[i, :c] = ids[sum(need[:i]):][:c]
    kc, vc = make_cache(gen, sum(need) + 2, ps, 3, d, TYPES[dt], layout, layers)
    want = [kc.clone(), vc.clone()]
    for i, p in enumerate(paths):
        for to, node in enumerate(p):
            if node < 0 or lens[i] < 0:
                break
            for w, old in zip(want, (kc, vc)):
                src, dst = lens[i] + node, lens[i] + to
                w[..., int(table[i, dst // ps]), dst % ps, :, :] = old[..., int(table[i, src // ps]), src % ps, :, :]
    got = sh.spechub_cache_accept(kc, vc, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                  torch.tensor(paths, dtype=torch.int32, device="cuda"), n)
    assert got["lens"].tolist() == [5, 12, 1023, -1, 14, 35, 8] and got["status"].tolist() == [0] * len(lens)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


def test_accept_of_a_long_path(sh):
    """Every second node of a chain of 1400, in more than one piece."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    n = 1400
    kc, vc = make_cache(gen, 90, 16, 2, 64, torch.bfloat16)
    table = torch.randperm(90, generator=gen, device="cuda").int()[None]
    flat = lambda c: c[table[0].long()].flatten(0, 1)  # noqa: E731
    old = flat(kc).clone(), flat(vc).clone()
    path = torch.arange(0, n, 2, dtype=torch.int32, device="cuda")[None]
    got = sh.spechub_cache_accept(kc, vc, table, torch.tensor([9], dtype=torch.int32, device="cuda"), path, n)
    assert got["lens"].tolist() == [9 + n // 2] and got["status"].tolist() == [0]
    for c, o in zip((kc, vc), old):
        assert torch.equal(flat(c)[9:9 + n // 2], o[9:9 + n:2])
        assert torch.equal(flat(c)[:9], o[:9]) and torch.equal(flat(c)[9 + n // 2:], o[9 + n // 2:])


def test_accept_stops_at_what_no_walk_leaves(sh):
    gen = torch.Generator(device="cuda").manual_seed(6)
    kc, vc = make_cache(gen, 8, 8, 1, 64, torch.bfloat16)
    table = torch.arange(8, dtype=torch.int32, device="cuda").reshape(4, 2)
    table[3, 1] = 99
    lens = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    paths = torch.tensor([[0, 2, 7], [0, 2, 2], [0, 0, 1], [0, 2, 6]], dtype=torch.int32, device="cuda")
    old = kc.clone()
    got = sh.spechub_cache_accept(kc, vc, table, lens, paths, 7)
    assert got["status"].tolist() == [256, 256, 256, 128] and got["lens"].tolist() == [2, 3, 3, 6]
    old[0, 1], old[2, 2] = old[0, 2].clone(), old[2, 3].clone()
    old[6, 4] = old[6, 5].clone()      # (slot 3 + 2 to slot 3 + 1; slot 9 lies on the page that is none)
    assert torch.equal(kc, old)


def test_refusals(sh):
    c = Case(16, [10, 20], 3, 2, 2, 64, 16)
    ok = dict(q=c.q, k_cache=c.kc, v_cache=c.vc, pages=c.pages, lens=c.lens, mask=c.mask)
    for bad in (dict(q=c.q.float()), dict(q=c.q[0]), dict(q=c.q[:1]), dict(q=c.q[..., :32]), dict(k_cache=c.kc.float()), dict(v_cache=c.vc[:1]),
                dict(pages=c.pages.long()), dict(pages=c.pages[:1]), dict(lens=c.lens.long()), dict(lens=c.lens.cpu()), dict(mask=c.mask[:2]),
                dict(mask=c.mask.repeat(1, 2)), dict(mask=c.mask[None]), dict(shared_pages=c.pages), dict(out=dict(out=c.q, lse=c.lens, status=c.lens))):
        with pytest.raises(ValueError):
            sh.spechub_tree_attention(**{**ok, **bad})
    for bad, code in ((dict(scale=0.0), -15), (dict(shared_len=1), -14), (dict(q=torch.zeros((2, 3, 3, 64), dtype=c.dt, device="cuda")), -12),
                      (dict(q=torch.zeros((2, 3, 4, 68), dtype=c.dt, device="cuda")[..., :64]), -11)):
        with pytest.raises(sh.SpecHubError) as e:
            sh.spechub_tree_attention(**{**ok, **bad})
        assert e.value.code == code
    odd = torch.zeros((4, 12, 1, 64), dtype=c.dt, device="cuda")
    with pytest.raises(sh.SpecHubError) as e:
        sh.spechub_cache_accept(odd, odd, c.pages, c.lens, c.pages)
    assert e.value.code == -12
    empty = sh.spechub_tree_attention(c.q[:0], c.kc, c.vc, c.pages[:0], c.lens[:0], c.mask)
    assert empty["out"].shape == (0, 3, 4, 64)


# ---- the operators together, as a decoding loop uses them -----------------------------------------------------------

def test_a_decoding_loop(sh):
    """Draft, append, attention, verification, walk and accept for some iterations: what the attention gives for the root's
    path is what attention over the emitted tokens gives in 64 bits, from scratch, at every iteration and layer."""
    B, n, V, hk, g, d, ps, layers, shared = 5, 15, 512, 2, 2, 64, 16, 2, 37
    gen = torch.Generator(device="cuda").manual_seed(11)
    dt, u = torch.bfloat16, 2.0 ** -8
    emb_k, emb_v = (torch.randn((layers, V, hk, d), generator=gen, device="cuda").to(dt) for _ in range(2))
    emb_q = torch.randn((layers, V, hk * g, d), generator=gen, device="cuda").to(dt)
    head = torch.randn((hk * g * d, V), generator=gen, device="cuda") * 0.2
    freq = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    tree = sh.Tree.heap(n)
    tab = sh.spechub_tree_tables(tree, n)
    kc, vc = make_cache(gen, 200, ps, hk, d, dt, layers=layers, fill=math.nan)
    order = torch.randperm(200, generator=gen, device="cuda").int()
    shared_pages, pages = order[:3].contiguous(), order[3:3 + B * 8].reshape(B, 8).contiguous()
    prefix = torch.randint(0, V, (shared,), generator=gen, device="cuda")
    for l in range(layers):   # the prefix is a chunk of a prompt of one sequence
        sh.spechub_cache_append(None, emb_k[l][prefix][None], emb_v[l][prefix][None], kc[l], vc[l], shared_pages[None].contiguous(),
                                torch.zeros(1, dtype=torch.int32, device="cuda"), None, freq)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    root = torch.randint(0, V, (B,), generator=gen, device="cuda")
    said = [[] for _ in range(B)]     # tokens in the cache
    moved = 0
    for it in range(6):
        un = torch.rand((B, n, 5), generator=gen, device="cuda")
        draft = torch.randn((B, n, V), generator=gen, device="cuda")
        tokens = sh.spechub_draft_sample(draft, un, tree)["tokens"].long()
        ids = torch.empty((B, n), dtype=torch.long, device="cuda")
        ids[:, 0] = root
        for m in range(1, n):
            ids[:, m] = tokens[:, (m - 1) // 2, (m - 1) % 2]
        hidden = []
        for l in range(layers):
            q = sh.spechub_cache_append(emb_q[l][ids], emb_k[l][ids], emb_v[l][ids], kc[l], vc[l], pages, lens, tab["depth"], freq,
                                        pos_offset=shared)["q"]
            r = sh.spechub_tree_attention(q, kc[l], vc[l], pages, lens, tab["mask"], shared_pages=shared_pages, shared_len=shared)
            assert r["status"].tolist() == [0] * B
            hidden.append((q, r["out"]))
        target = hidden[-1][1].reshape(B, n, -1).float() @ head
        out = sh.spechub_verify_tree(target, draft, tokens.int(), un, tree)
        path, emitted = out["path_nodes"], out["path_tokens"]
        new = sh.spechub_cache_accept(kc, vc, pages, lens, path, n)
        assert new["status"].tolist() == [0] * B
        for b in range(B):
            nodes = [x for x in path[b].tolist() if x >= 0]
            said[b] += [int(ids[b, x]) for x in nodes]
            moved += sum(x != i for i, x in enumerate(nodes))
            assert int(new["lens"][b]) == len(said[b])
            seq = torch.cat((prefix, torch.tensor(said[b], device="cuda")))
            pos = torch.arange(len(seq), device="cuda").double()
            for l in range(layers):
                k64, mag = rotate64(emb_k[l][seq].double(), pos, freq.double(), False)
                mine = kc[l][pages[b].long()].flatten(0, 1)[: len(said[b])].double()
                assert bool(((mine - k64[shared:]).abs() <= u * k64[shared:].abs() * (1 + 1e-6) + 6e-7 * mag[shared:]).all())
                k64 = k64.to(dt).double()      # (what is in the cache is rounded)
                k64[shared:] = mine
                k64[:shared] = kc[l][shared_pages.long()].flatten(0, 1)[:shared].double()
                v64 = emb_v[l][seq].double()
                q, got = hidden[l]
                for i, x in enumerate(nodes):
                    upto = shared + len(said[b]) - len(nodes) + i + 1
                    for h in range(hk * g):
                        s = (k64[:upto, h // g] @ q[b, x, h].double()) * d ** -0.5
                        p = torch.softmax(s, 0)
                        want, mags = p @ v64[:upto, h // g], p @ v64[:upto, h // g].abs()
                        assert bool(((got[b, x, h].double() - want).abs() <= u * want.abs() + (u + 1e-3) * mags).all()), (it, b, l, i)
        lens = new["lens"]
        last = out["n_emitted"].long() - 1
        root = emitted.gather(1, last[:, None])[:, 0].long()
    assert moved > 5


def test_too_many_query_heads_per_cache_head(sh):
    c = Case(2, [5, 6], 3, 1, 4, 64, 16)
    for heads, code in ((129, -12), (4096, -12)):
        with pytest.raises(sh.SpecHubError) as e:
            sh.spechub_tree_attention(torch.zeros((2, 3, heads, 64), dtype=c.dt, device="cuda"), c.kc, c.vc, c.pages, c.lens, c.mask)
        assert e.value.code == code
