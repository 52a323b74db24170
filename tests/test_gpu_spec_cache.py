"""The cache's side of a speculative step: append with norms and rotation, accepted paths, reading back."""
import numpy as np
import pytest

import paper_2507_17769_b200 as ps
from spec_util import PAGE, Cache

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (3, 3, 128), (8, 1, 128), (8, 8, 64), (2, 1, 64), (40, 20, 64)]


def angles(positions, rot, theta=10000.0):
    """float32 [positions, rot]: cosines, then sines."""
    import torch

    freq = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return torch.cat([a.cos(), a.sin()], dim=1).float().cuda()


def turned(x, weight, eps, table, pos, interleaved):
    """(the definition in 64 bits, what fp32 arithmetic may add to a result's own rounding).

    In fp32 a normed element carries some 2^-21 relative (a sum of d squares pairwise and in lanes, rsqrt, two products), a rotated one the
    sum of both of its pair's plus three roundings: 2^-20 of |a cos| + |b sin| bounds it."""
    import torch

    y = x.double()
    if weight is not None:
        y = y / (y.pow(2).mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    mag = y.abs()
    if table is not None:
        h = table.size(1) // 2
        c, s = table[pos].double()[:, None, :h], table[pos].double()[:, None, h:]
        i = torch.arange(h, device=x.device)
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        a, b = y[..., ia], y[..., ib]
        y, mag = y.clone(), mag.clone()
        y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
        mag[..., ia] = mag[..., ib] = (a.abs() + b.abs())
    return y, mag * 2.0 ** -20


def check_rounded(got, want, slack):
    over = (got.double() - want).abs() - (2.0 ** -8 * want.abs() * (1 + 2.0 ** -8) + slack)
    assert float(over.max()) <= 0, "%.3e over half a step" % float(over.max())


def check_fp8(codes, scale, want, slack):
    """A scale is the largest magnitude / 448 rounded up to 8 significant bits; a code is the nearest to its value over the scale."""
    import torch

    amax = want.abs().amax(-1)
    s = scale.double()
    zero = amax == 0
    assert torch.equal(s[zero], torch.ones_like(s[zero]))
    near = slack.amax(-1) / 448
    assert bool((s[~zero] >= (amax / 448 - near)[~zero]).all()) and bool((s <= (amax / 448 + near) * (1 + 2.0 ** -7))[~zero].all())
    assert int((scale.view(torch.int32) & 0xFFFF).abs().sum()) == 0
    got = codes.view(torch.float8_e4m3fn).double() * s[..., None]
    over = (got - want).abs() - (torch.maximum(want.abs(), s[..., None] * 2.0 ** -6) * 2.0 ** -4 * (1 + 2.0 ** -20) + slack)
    assert float(over.max()) <= 0


def append(heads, prior, q_len, rot, interleaved=False, norm=True, fp8=False, positions=None, stride_extra=0, in_place=False, seed=0, eps=1e-6):
    import torch

    hq, hkv, d = heads
    prior, q_len = np.asarray(prior, dtype=np.int32), np.asarray(q_len, dtype=np.int32)
    c = Cache(hq, hkv, d, prior + q_len, seed=seed, fp8=fp8)
    T = int(q_len.sum())
    fused = c.normal(T, (hq + 2 * hkv) * d + stride_extra, scale=3.0)
    x = fused[:, :(hq + 2 * hkv) * d].unflatten(1, (hq + 2 * hkv, d))
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if in_place:
        q = q.contiguous()
    q_in = q.clone()
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(prior, q_len)])
    if positions is not None:
        pos = positions(pos)
    table = angles(int(pos.max()) + 1, rot) if rot else None
    qw, kw = ((1 + 0.3 * torch.randn(d, generator=c.gen, device="cuda")).bfloat16() for _ in range(2)) if norm else (None, None)
    pos = torch.from_numpy(pos.astype(np.int32)).cuda()
    got = c.pa.write_rope(q, k, v, c.table, prior, q_len, table, positions=pos if positions is not None else None, q_weight=qw, k_weight=kw, eps=eps,
                          interleaved=interleaved, q_out=q if in_place else None)
    c.pa.check_pool()
    assert (got.data_ptr() == q.data_ptr()) == in_place
    check_rounded(got, *turned(q_in, qw, eps, table, pos.long(), interleaved))
    want, slack = turned(k, kw, eps, table, pos.long(), interleaved)
    t = 0
    for r, n in enumerate(q_len):
        s, p = slice(t, t + int(n)), slice(int(prior[r]), int(prior[r] + n))
        if fp8:
            kc, vc, ks, vs = c.pa.gather_fp8(c.table[r], int(prior[r] + n))
            check_fp8(kc[p], ks[p], want[s], slack[s])
            check_fp8(vc[p], vs[p], v[s].double(), torch.zeros_like(want[s]))
        else:
            gk, gv = c.pa.gather(c.table[r], int(prior[r] + n))
            check_rounded(gk[p], want[s], slack[s])
            assert torch.equal(gv[p], v[s])
        t += int(n)
    return c, x, got


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_append_with_norms_and_rotation(heads, interleaved, norm):
    append(heads, [0, 17, 100, 5], [1, 33, 2, 1], heads[2], interleaved, norm)


@pytest.mark.parametrize("rot", [0, 16, 48, 64])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_of_a_head_is_rotated(rot, interleaved):
    for heads in ((32, 8, 128), (4, 2, 64)):
        append(heads, [3, 40], [20, 1], rot, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads", [(64, 8, 128), (1, 1, 128)])
def test_append_quantised(heads, interleaved):
    append(heads, [0, 31, 16], [40, 1, 9], 128, interleaved, fp8=True)
    append(heads, [0, 31, 16], [40, 1, 9], 64, interleaved, norm=False, fp8=True)


def test_positions_strides_and_in_place():
    append((32, 8, 128), [0, 50], [30, 7], 128, positions=lambda p: 4000 - 3 * p, stride_extra=8)
    append((8, 8, 64), [9], [1], 64, stride_extra=64)
    append((32, 8, 128), [12], [25], 128, in_place=True)


@pytest.mark.parametrize("n", [64, 65, 513, 4001, 8100])
def test_batches_of_many_requests(n):
    rng = np.random.default_rng(n)
    append((2, 1, 64), rng.integers(0, 20, n), rng.integers(1, 3, n), 64, seed=n)


def test_without_norm_and_rotation_it_is_write():
    import torch

    for fp8 in (False, True):
        c, x, q = append((4, 2, 128), [0, 8], [21, 5], 0, norm=False, fp8=fp8)
        other = ps.PagedAttention(4, 2, 128, c.num_pages, poison=True, kv_dtype=int(fp8))
        other.write(x[:, 4:6].contiguous(), x[:, 6:].contiguous(), c.table, [0, 8], [21, 5])
        n = c.pa.pool.numel() - 1024
        offset = lambda p: (p.pool.data_ptr() + 1023) // 1024 * 1024 - p.pool.data_ptr()  # noqa: E731
        a, b = (p.pool[offset(p):offset(p) + n] for p in (c.pa, other))
        assert torch.equal(a, b) and torch.equal(q, x[:, :4])


def test_extreme_values_are_normed_and_quantised():
    """Zero heads (a norm of eps alone, a scale of 1), the largest and the smallest magnitudes that fp32 squares hold, infinities and NaN."""
    import torch

    for fp8 in (False, True):
        c = Cache(2, 1, 128, [8], fp8=fp8)
        x = c.normal(8, 4, 128)
        x[0], x[1], x[2] = 0, x[1] * 1e15, x[2] * 1e-15
        x[3, :, 5] = float("inf")
        x[4, :, 7] = float("nan")
        w = torch.ones(128, device="cuda", dtype=torch.bfloat16)
        q = c.pa.write_rope(x[:, :2], x[:, 2:3], x[:, 3:], c.table, [0], [8], None, q_weight=w, k_weight=w, eps=1e-6)
        c.pa.check_pool()
        want, slack = turned(x[:, :3], w, 1e-6, None, None, False)
        check_rounded(q[[0, 1, 2, 5, 6, 7]], want[[0, 1, 2, 5, 6, 7], :2], slack[[0, 1, 2, 5, 6, 7], :2])
        assert bool(torch.isnan(q[3, :, 5]).all()) and bool(torch.isnan(q[4]).all()) and float(q[3, :, :5].abs().max()) == 0
        k, v = c.pa.read(c.table, [0], [8])
        assert float(k[0].abs().max()) == 0 and float(v[0].abs().max()) == 0 and bool(torch.isfinite(k[[0, 1, 2, 5, 6, 7]]).all())
        assert bool(torch.isnan(v[4, 0, 7])) and (fp8 or torch.equal(v[3], x[3, 3:]))


def test_pages_and_positions_outside_are_skipped_and_reported():
    import torch

    c = Cache(2, 1, 64, [16, 16, 16])
    x = c.normal(3, 4, 64)
    table = c.table.clone()
    table[0, 0] = c.num_pages
    table[1, 0] = -3
    cs = angles(8, 64)
    pos = torch.tensor([1, 2, 8], dtype=torch.int32, device="cuda")
    before = c.pa.pool.clone()
    out = torch.full((3, 2, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    for bad in (pos, torch.tensor([1, 2, -1], dtype=torch.int32, device="cuda")):
        c.pa.write_rope(x[:, :2], x[:, 2:3], x[:, 3:], table, [0, 0, 0], [1, 1, 1], cs, positions=bad, q_out=out)
        with pytest.raises(ps.PsError) as e:
            c.pa.check_pool()
        assert e.value.status == ps.binding.PS_ERR_BOUNDS
        assert torch.equal(before, c.pa.pool) and bool((out == 7).all())
    c.pa.check_pool()  # the report is given once


# ---------------------------------------------------------------------------


def paths(n_nodes, width, rng, least=0):
    index = np.full((len(n_nodes), width), -7, dtype=np.int32)  # (what stands behind a path is not looked at)
    count = np.zeros(len(n_nodes), dtype=np.int32)
    for r, n in enumerate(n_nodes):
        count[r] = rng.integers(least, min(n, width) + 1)
        index[r, :count[r]] = np.sort(rng.choice(n, count[r], replace=False))
    return index, count


@pytest.mark.parametrize("heads,fp8", [((32, 8, 128), False), ((32, 8, 128), True), ((3, 3, 128), False), ((8, 8, 64), False), ((1, 1, 64), False), ((1, 1, 128), True)])
@pytest.mark.parametrize("n", [1, 7, 70, 600])
def test_accepted_paths(heads, fp8, n):
    import torch

    rng = np.random.default_rng(n)
    prior, nodes = rng.integers(0, 100, n).astype(np.int32), rng.integers(1, 65 if n < 600 else 12, n).astype(np.int32)
    c = Cache(*heads, prior + nodes, seed=n, fp8=fp8).fill()
    index, count = paths(nodes, int(nodes.max()), rng)
    if n > 1:
        index[0, :nodes[0]], count[0] = np.arange(nodes[0]), nodes[0]  # the whole tree, a chain: nothing moves
        index[1, 0], count[1] = nodes[1] - 1, 1
    c.pa.accept(c.table, prior, nodes, torch.from_numpy(index).cuda(), torch.from_numpy(count).cuda())
    c.pa.check_pool()
    for r in range(n):
        p, m = int(prior[r]), int(count[r])
        for x, got in zip((c.k[r], c.v[r]), c.stored(r)):
            want = x.clone()
            want[p:p + m] = x[p + torch.from_numpy(index[r, :m].astype(np.int64)).cuda()]
            assert torch.equal(want, got)


def test_long_paths_move_in_order():
    """Every destination but the last is the source of an earlier token: what is read must not have been overwritten."""
    import torch

    nodes = 250
    for fp8 in (False, True):
        c = Cache(2, 2, 128, [5 + nodes], fp8=fp8).fill()
        index = torch.arange(1, nodes, dtype=torch.int32, device="cuda")[None].contiguous()
        c.pa.accept(c.table, [5], [nodes], index, torch.tensor([nodes - 1], dtype=torch.int32, device="cuda"))
        c.pa.check_pool()
        for x, got in zip((c.k[0], c.v[0]), c.stored(0)):
            assert torch.equal(got[:5], x[:5]) and torch.equal(got[5:5 + nodes - 1], x[6:]) and torch.equal(got[-1], x[-1])


@pytest.mark.parametrize("path,count", [([0, 2, 2], 3), ([0, 3, 2], 3), ([1, 2, 9], 3), ([-1, 1, 2], 3), ([0, 1, 2], 4), ([0, 1, 2], -1), ([0, 0, 0], 3)])
def test_what_is_no_path_leaves_its_request_as_it_is(path, count):
    import torch

    c = Cache(2, 2, 64, [20, 20]).fill()
    index = torch.tensor([path, [1, 3, 5]], dtype=torch.int32, device="cuda")
    c.pa.accept(c.table, [11, 11], [9, 9], index, torch.tensor([count, 3], dtype=torch.int32, device="cuda"))
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_BOUNDS
    assert all(torch.equal(a, b) for a, b in zip(c.stored(0), (c.k[0], c.v[0])))
    assert torch.equal(c.stored(1)[0][11:14], c.k[1][[12, 14, 16]])


def test_paths_through_pages_outside_are_skipped():
    import torch

    c = Cache(2, 2, 64, [40]).fill()
    table = c.table.clone()
    table[0, 1] = c.num_pages + 4
    c.pa.accept(table, [8], [32], torch.tensor([[3, 10, 25]], dtype=torch.int32, device="cuda"), torch.tensor([3], dtype=torch.int32, device="cuda"))
    with pytest.raises(ps.PsError):
        c.pa.check_pool()
    k = c.k[0].clone()
    k[8], k[10] = c.k[0][11], c.k[0][33]  # (node 10 lies at 18, on the page outside)
    assert torch.equal(c.stored(0)[0], k)


# ---------------------------------------------------------------------------


@pytest.mark.parametrize("heads,fp8", [((32, 8, 128), False), ((32, 8, 128), True), ((20, 20, 128), False), ((9, 9, 128), True), ((8, 8, 64), False), ((3, 3, 64), False)])
@pytest.mark.parametrize("n", [1, 5, 65, 520])
def test_read_back(heads, fp8, n):
    import torch

    rng = np.random.default_rng(n)
    kv_len = rng.integers(1, 200 if n < 500 else 30, n).astype(np.int32)
    c = Cache(*heads, kv_len, seed=n, fp8=fp8).fill()
    begin = np.array([rng.integers(0, x + 1) for x in kv_len], dtype=np.int32)
    length = np.array([rng.integers(0, x - b + 1) for x, b in zip(kv_len, begin)], dtype=np.int32)
    for lo, cnt in ((begin, length), (np.zeros_like(kv_len), kv_len), (begin, np.zeros_like(length))):
        k, v = c.pa.read(c.table, lo, cnt)
        c.pa.check_pool()
        assert k.shape == v.shape == (int(cnt.sum()), heads[1], heads[2])
        for got, parts in ((k, c.k), (v, c.v)):
            want = torch.cat([x[int(a):int(a + b)] for x, a, b in zip(parts, lo, cnt)]).to(torch.bfloat16)
            assert torch.equal(got, want)


def test_read_back_outside_the_pool_is_left_and_reported():
    import torch

    c = Cache(2, 2, 64, [40]).fill()
    table = c.table.clone()
    table[0, 1] = -1
    k, v = (torch.full((40, 2, 64), 5.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    ps.ps_kv_read(c.pa.kv, table, table.size(1), [0], [40], k, None, torch.cuda.current_stream().cuda_stream)
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_BOUNDS
    assert bool((k[16:32] == 5).all()) and torch.equal(k[:16], c.k[0][:16]) and torch.equal(k[32:], c.k[0][32:]) and bool((v == 5).all())


def test_outputs_on_a_16_byte_boundary():
    import torch

    for fp8 in (False, True):
        c = Cache(2, 2, 128, [50], fp8=fp8).fill()
        room = torch.empty(2, 50 * 256 + 8, device="cuda", dtype=torch.bfloat16)
        k, v = (room[i, 8:].view(50, 2, 128) if (room[i, 8:].data_ptr() & 31) else room[i, :-8].view(50, 2, 128) for i in range(2))
        ps.ps_kv_read(c.pa.kv, c.table, c.table.size(1), [0], [50], k, v, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(k, c.k[0].bfloat16()) and torch.equal(v, c.v[0].bfloat16())


def test_offsets_beyond_32_bits():
    """Pages at the end of a pool of more than 4 GB (and 2^31 elements)."""
    import torch

    pages = 150000  # x 32 KB: 4.9 GB
    pa = ps.PagedAttention(4, 4, 128, pages)
    last = torch.arange(pages - 4, pages, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((64, 12, 128), generator=g, device="cuda").bfloat16()
    q = pa.write_rope(x[:, :4], x[:, 4:8], x[:, 8:], last, [0], [64], None)
    k, v = pa.read(last, [0], [64])
    assert torch.equal(k, x[:, 4:8]) and torch.equal(v, x[:, 8:])
    mask = torch.full((64, 1), -1, dtype=torch.int64, device="cuda")
    out, _ = pa.run_tree(q, last, mask, [0], [64])
    pa.accept(last, [0], [64], torch.tensor([[9, 60]], dtype=torch.int32, device="cuda"), torch.tensor([2], dtype=torch.int32, device="cuda"))
    assert torch.equal(pa.read(last, [0], [2])[0], x[[9, 60], 4:8])
    pa.check_pool()
    s = torch.einsum("qhd,khd->hqk", q.double(), x[:, 4:8].double()) / 128 ** 0.5
    want = torch.einsum("hqk,khd->qhd", s.softmax(-1), x[:, 8:].double())
    assert float((out.double() - want).abs().max()) < 0.05  # (a wrong page is off by whole values)


assert PAGE == 16
