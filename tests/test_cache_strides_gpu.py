"""The cache operators' strides and lengths at their limits: tensors whose strides do not nest, that lie over themselves or between
each other; the largest length."""
import gc

import pytest

from test_cache_gpu import Case, make_cache, sh, tree_mask  # noqa: F401  (sh: the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def nothing_left():
    """The modules behind this one find the device's memory as it was: frames that an exception's traceback keeps alive go, too."""
    yield
    gc.collect()
    torch.cuda.empty_cache()


def test_outputs_whose_strides_do_not_nest(sh):
    """Rows 0, 2, 4 of one node lie between rows 3, 5, 7 of the next: unusual, but apart."""
    n, h, d = 2, 3, 64
    c = Case(1, [100, 40, -1, 300], n, 1, h, d, 16, shared=50, mask=tree_mask(n))
    want = c.run(sh)
    c.check(want)
    room = torch.full((4 * 8 * d,), 3.0, dtype=c.dt, device="cuda")
    view = room.as_strided((4, n, h, d), (8 * d, 3 * d, 2 * d, 1))
    c.run(sh, out=dict(out=view, lse=want["lse"].clone(), status=want["status"].clone()))
    for i in (0, 1, 3):
        assert torch.equal(view[i], want["out"][i])
    assert bool((view[2] == 3.0).all())
    freq = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    k = torch.randn((4, n, 1, d), generator=c.gen, device="cuda").to(c.dt)
    turned = sh.spechub_cache_append(c.q, k, k, c.kc, c.vc, c.pages, c.lens, None, freq)["q"].clone()
    sh.spechub_cache_append(c.q, k, k, c.kc, c.vc, c.pages, c.lens, None, freq, q_out=view)
    for i in (0, 1, 3):
        assert torch.equal(view[i], turned[i])


def test_outputs_and_caches_over_themselves_are_refused(sh):
    n, h, d = 2, 3, 64
    c = Case(2, [10, 20], n, 1, h, d, 16, mask=tree_mask(n))
    room = torch.zeros((1 << 16,), dtype=c.dt, device="cuda")
    lse, status = torch.empty((2, n, h), device="cuda"), torch.empty((2,), dtype=torch.int32, device="cuda")
    for strides in ((8 * d, d, d, 1), (8 * d, 2 * d, d, 1), (5 * d, 3 * d, d, 1)):
        view = room.as_strided((2, n, h, d), strides)
        with pytest.raises(sh.SpecHubError) as e:
            c.run(sh, out=dict(out=view, lse=lse, status=status))
        assert e.value.code == -11
        with pytest.raises(sh.SpecHubError) as e:
            sh.spechub_cache_append(c.q, c.q[:, :, :1], c.q[:, :, :1], c.kc, c.vc, c.pages, c.lens, q_out=view)
        assert e.value.code == -11
    over = room.as_strided((8, 16, 1, d), (8 * d, d, d, 1))
    path = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    with pytest.raises(sh.SpecHubError) as e:
        sh.spechub_cache_accept(over, room[1 << 15:].as_strided((8, 16, 1, d), (16 * d, d, d, 1)), c.pages, c.lens, path, n)
    assert e.value.code == -11
    assert bool((room == 0).all())


def test_slices_of_one_tensor_side_by_side(sh):
    """Queries, outputs, keys and values that lie between each other in one tensor share nothing, and are taken."""
    b, n, hk, g, d = 3, 5, 2, 2, 64
    c = Case(3, [30, 0, 200], n, hk, g, d, 16, mask=tree_mask(n))
    want = c.run(sh)
    c.check(want)
    h = hk * g
    room = torch.full((b, n, 2 * h + 2 * hk, d), 3.0, dtype=c.dt, device="cuda")
    q, out, k, v = room[:, :, :h], room[:, :, h:2 * h], room[:, :, 2 * h:2 * h + hk], room[:, :, 2 * h + hk:]
    q.copy_(c.q)
    got = sh.spechub_tree_attention(q, c.kc, c.vc, c.pages, c.lens, c.mask, out=dict(out=out, lse=want["lse"].clone(), status=want["status"].clone()))
    assert torch.equal(got["out"], want["out"]) and torch.equal(q, c.q) and bool((k == 3.0).all())
    freq = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
    turned = sh.spechub_cache_append(c.q, k.clone(), v.clone(), c.kc, c.vc, c.pages, c.lens, None, freq)["q"]
    sh.spechub_cache_append(q, k, v, c.kc, c.vc, c.pages, c.lens, None, freq, q_out=out)
    assert torch.equal(out, turned) and torch.equal(q, c.q)
    sh.spechub_cache_append(q, k, v, c.kc, c.vc, c.pages, c.lens, None, freq, q_out=q)
    assert torch.equal(q, turned)
    for bad in (room[:, :, 1:h + 1], room[:, :, h + 1:2 * h + 1]):
        with pytest.raises(sh.SpecHubError) as e:
            sh.spechub_cache_append(q, k, v, c.kc, c.vc, c.pages, c.lens, None, freq, q_out=bad)
        assert e.value.code == -11
    with pytest.raises(sh.SpecHubError) as e:
        sh.spechub_tree_attention(q, c.kc, c.vc, c.pages, c.lens, c.mask, out=dict(out=room[:, :, 1:h + 1], lse=want["lse"], status=want["status"]))
    assert e.value.code == -11


def test_accept_of_keys_and_values_in_one_tensor(sh):
    """Heads of keys and of values in turn, and one behind the other; the same tensor twice is refused."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    table, lens = torch.tensor([[2, 0], [1, 3]], dtype=torch.int32, device="cuda"), torch.tensor([3, 12], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 2, 5], [0, 1, 3]], dtype=torch.int32, device="cuda")
    kv = torch.randn((3, 4, 16, 4, 64), generator=gen, device="cuda").bfloat16()
    want = kv.clone()
    for i in range(2):
        for to, node in enumerate(path[i].tolist()):
            src, dst = int(lens[i]) + node, int(lens[i]) + to
            want[:, int(table[i, dst // 16]), dst % 16] = kv[:, int(table[i, src // 16]), src % 16]
    for k, v in ((slice(0, None, 2), slice(1, None, 2)), (slice(0, 2), slice(2, 4))):
        got = kv.clone()
        r = sh.spechub_cache_accept(got[..., k, :], got[..., v, :], table, lens, path, 7)
        assert r["lens"].tolist() == [6, 15] and r["status"].tolist() == [0, 0]
        assert torch.equal(got, want)
    with pytest.raises(sh.SpecHubError) as e:
        sh.spechub_cache_accept(kv, kv, table, lens, path, 7)
    assert e.value.code == -11


def test_accept_at_the_largest_length(sh):
    """Far behind the table: nothing moves, and the sequence does not become one that is absent."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    kc, vc = make_cache(gen, 4, 8, 1, 64, torch.bfloat16)
    old = kc.clone(), vc.clone()
    lens = torch.tensor([2147483647, 2147483646, 2147483640], dtype=torch.int32, device="cuda")
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None].expand(3, 4).contiguous()
    path = torch.tensor([[0, 2, 6]] * 3, dtype=torch.int32, device="cuda")
    got = sh.spechub_cache_accept(kc, vc, table, lens, path, 7)
    assert got["lens"].tolist() == [2147483647, 2147483647, 2147483643] and got["status"].tolist() == [128] * 3
    assert torch.equal(kc, old[0]) and torch.equal(vc, old[1])


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("d,shared,n", [(64, 0, 1), (128, 200, 33)])
def test_scores_of_the_largest_magnitude(sh, d, shared, n, sign, dt):
    """Scores of 2^25, exact in 32 bits, at every third key and below it by 2^18 at the others: all weight is at those keys.
    Their weights are equal, whatever the reference is rounded to: out is their values' mean, off by the common rounding of the weights and its
    own (2 u |out|) and by the sums' (n 2^-23 of the values); lse by half the spacing of 2^26 twice, the second time by ln 2."""
    c = Case(23, [500, 3, 260], n, 1, 4, d, 16, dt, shared=shared, mask=tree_mask(n), q_sd=0.0)
    c.q[..., 0] = 4096.0
    for pages, count in [(c.ids_shared, shared)] + [(c.table[i], x + n) for i, x in enumerate(c.lens_list)]:
        for at in range(count):
            key = c.kc[int(pages[at // 16]), at % 16]
            key[:] = 0
            key[..., 0] = sign * 8192.0 if at % 3 == 0 else sign * 8192.0 - 64.0
    got = c.run(sh, scale=1.0)
    assert got["status"].tolist() == [0, 0, 0]
    u = torch.finfo(c.dt).eps / 2
    for i, x in enumerate(c.lens_list):
        k = torch.cat((c.flat(c.kc, c.ids_shared, shared), c.flat(c.kc, c.table[i], x + n)))[:, 0, 0]
        v = torch.cat((c.flat(c.vc, c.ids_shared, shared), c.flat(c.vc, c.table[i], x + n)))[:, 0]
        sees = torch.ones((n, len(k)), dtype=torch.bool, device="cuda")
        sees[:, shared + x:] = torch.from_numpy(c.sees).cuda()
        top = torch.where(sees, k, -1e9).amax(1)
        hit = (sees & (k == top[:, None])).double()
        want = hit @ v / hit.sum(1, keepdim=True)
        far = (got["out"][i].double() - want[:, None]).abs()
        assert bool((far <= 2 * u * want[:, None].abs() + len(k) * 2.0 ** -23 * v.abs().max() + (2.0 ** -25 if dt == "fp16" else 0)).all())
        lse = top * 4096 + hit.sum(1).log()
        assert bool(((got["lse"][i].double() - lse[:, None]).abs() <= 2 + 2 * 0.7).all())
