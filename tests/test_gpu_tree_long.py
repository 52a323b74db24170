"""What loose bounds on long contexts would let through: every key tile's V has its own mark, and K that is not finite reaches the rows that see it."""
import math

import numpy as np
import pytest

from spec_util import Cache, check_tree, tree_masks, tree_reference

pytestmark = pytest.mark.gpu

TILE = 128
LONG = [((4, 1, 128), False, [60000], [40]), ((2, 2, 64), False, [60000], [40]), ((4, 1, 128), True, [60000], [40]), ((8, 1, 128), False, [20000, 9000], [64, 7]),
        ((8, 1, 128), True, [20000, 9000], [64, 7]), ((4, 2, 64), False, [15000, 100], [256, 3])]


def marked(c):
    """V is zero but for element (tile % d) of every token of a key tile, 1 or 2."""
    import torch

    for r, n in enumerate(c.kv_len):
        tile = torch.arange(int(n), device="cuda") // TILE
        c.v[r].zero_()
        c.v[r][torch.arange(int(n), device="cuda"), :, tile % c.dim] = (1 + tile // c.dim % 2)[:, None].to(torch.bfloat16)


@pytest.mark.parametrize("heads,fp8,prior,nodes", LONG)
def test_each_key_tile_has_its_part(heads, fp8, prior, nodes):
    """An element of the output is the weight of the tiles that mark it, and so is sum |w v|, so the bounds of tree_reference are relative ones: some 2^-8
    + 2^-7 (FP8 2^-8 + 2^-10) of an element.  A tile that is lost or taken twice changes its element by a twelfth at the least (64 dimensions,
    eight tiles of 1 or 2); that check_tree sees one is shown on the reference."""
    import torch

    c = Cache(*heads, np.add(prior, nodes), seed=41, fp8=fp8)
    marked(c)
    c.fill()
    mask, sees = tree_masks(nodes, (max(nodes) + 63) // 64, np.random.default_rng(42))
    q = c.normal(sum(nodes), heads[0], heads[2], scale=0.25)  # (scores that leave each tile about its share of the weight)
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    ref, ref_lse, bound, lse_bound = tree_reference(c, q, prior, sees)
    if fp8:
        # (no weight lies in f16's subnormal range: scores of this spread are within 14 powers of two.  V's rounding to f16 is 2^-11 more.)
        bound = bound - 2.0 ** -13 + 2.0 ** -11 * ref.abs()
    check_tree(out, lse, (ref, ref_lse, bound, lse_bound))
    tiles = (int(c.kv_len[0]) - nodes[0]) // TILE
    for tile in (0, 1, tiles // 3, tiles - 1):
        v = c.v[0].clone()
        c.v[0][tile * TILE:(tile + 1) * TILE] = 0
        lost = tree_reference(c, q, prior, sees)[0]
        c.v[0] = v
        with pytest.raises(AssertionError):
            check_tree(out, lse, (lost, ref_lse, bound, lse_bound))


@pytest.mark.parametrize("heads,fp8,prior,nodes", LONG)
def test_long_contexts_to_the_spread_of_their_roundings(heads, fp8, prior, nodes):
    """Random V.  A weight's rounding is off by at most 2^-8 of it (FP8: 2^-11, as is V's in f16; below 2^-14 2^-25, where the largest is at least 1), either
    way, so n of them add up to t * sqrt(sum (c w v)^2) at the most, but for 2 exp(-t^2 / 2) of the elements: t = 7, 5e-11.  The scores' part and the output's own
    rounding are tree_reference's."""
    import torch

    c = Cache(*heads, np.add(prior, nodes), seed=43, fp8=fp8).fill()
    mask, sees = tree_masks(nodes, (max(nodes) + 63) // 64, np.random.default_rng(44))
    q = c.normal(sum(nodes), heads[0], heads[2])
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    ref, ref_lse, bound, lse_bound = tree_reference(c, q, prior, sees)
    group, t = heads[0] // heads[1], 0
    for r, s in enumerate(sees):
        n, p = nodes[r], prior[r]
        k, v = (x[r].double().repeat_interleave(group, dim=1).transpose(0, 1) for x in (c.k, c.v))
        score = q[t:t + n].double().transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(c.dim)
        score[:, :, p:] = score[:, :, p:].masked_fill(~torch.from_numpy(s).cuda(), -math.inf)
        w = (score - ref_lse[t:t + n].transpose(0, 1)[..., None]).exp()
        spread = (w.square() @ v.square()).sqrt() * (2.0 ** -10 if fp8 else 2.0 ** -8)
        if fp8:
            spread = spread + w.amax(-1, keepdim=True) * 2.0 ** -25 * v.square().sum(1, keepdim=True).sqrt()
        weight = (w @ v.abs()).transpose(0, 1)
        loose = (2.0 ** -11 if fp8 else 2.0 ** -7) * weight + (2.0 ** -13 if fp8 else 0.0)
        bound[t:t + n] += 7 * spread.transpose(0, 1) - loose
        t += n
    check_tree(out, lse, (ref, ref_lse, bound, lse_bound))


@pytest.mark.parametrize("heads,fp8", [((8, 2, 128), False), ((8, 8, 64), False), ((8, 1, 128), False), ((8, 2, 128), True)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_keys_that_are_not_finite(heads, fp8, value):
    """A row that sees a key with a NaN, or infinities that make its score NaN or +inf, is NaN; one whose scores are -inf there, or that does not see it, is
    as the others are (an FP8 cache's infinity takes its vector's scale with it: NaN)."""
    import torch

    prior, nodes = np.array([0, 250, 77], dtype=np.int32), np.array([20, 64, 100], dtype=np.int32)
    c = Cache(*heads, prior + nodes, seed=45, fp8=fp8)
    bad = ([3], [0, 40, 63], [99])
    for r in range(3):
        for i in bad[r]:
            c.k[r][prior[r] + i, :, 5] = value
    c.fill()
    mask, sees = tree_masks(nodes, 2, np.random.default_rng(46))
    q = c.normal(int(nodes.sum()), heads[0], heads[2])
    out, lse = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    clean = Cache(*heads, prior + nodes, seed=45, fp8=fp8)
    clean.k = [torch.nan_to_num(k, 0, 0, 0) for k in c.k]
    clean.v = c.v
    group, t = heads[0] // heads[1], 0
    for r, s in enumerate(sees):
        n = int(nodes[r])
        seen = torch.from_numpy(s).cuda()
        sums = torch.stack([q[t:t + n].double()[..., 5] * c.k[r][prior[r] + i].double().repeat_interleave(group, dim=0)[:, 5] for i in bad[r]], dim=-1)
        if fp8:
            sums = torch.full_like(sums, math.nan)
        lost = ((torch.isnan(sums) | (sums == math.inf)) & seen[:, None, bad[r]]).any(-1)  # [n, heads]
        a, b = out[t:t + n], lse[t:t + n]
        assert bool(torch.isnan(a[lost]).all()) and not bool(torch.isfinite(b[lost]).any())
        # the others: the bad keys unseen
        hidden = s.copy()
        hidden[:, bad[r]] = False
        want, want_lse, bound, lse_bound = (x[t:t + n] for x in tree_reference(clean, q, prior, [hidden if k == r else x for k, x in enumerate(sees)]))
        assert bool(lost.any()) and (r == 1 or not bool(lost.all()))
        if not bool(lost.all()):
            check_tree(a[~lost], b[~lost], (want[~lost], want_lse[~lost], bound[~lost], lse_bound[~lost]))
        t += n
