"""Append with norms and rotation where there are many tokens: stretches of tokens behind bulk copies."""
import numpy as np
import pytest

import paper_2507_17769_b200 as ps
from spec_util import Cache
from test_gpu_spec_cache import HEADS, angles, append, check_rounded, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,fp8", [(h, False) for h in HEADS] + [((32, 8, 128), True), ((1, 1, 128), True), ((64, 8, 128), True)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_many_tokens(heads, fp8, interleaved):
    append(heads, [0, 17, 100, 5, 31], [300, 1, 257, 419, 40], heads[2], interleaved, fp8=fp8, seed=3)


@pytest.mark.parametrize("tokens", [295, 296, 297, 299, 592, 593, 2369, 9501])
def test_counts_of_tokens(tokens):
    append((4, 2, 64), [7], [tokens], 32, seed=tokens)


@pytest.mark.parametrize("rot", [0, 16, 96])
@pytest.mark.parametrize("norm", [False, True])
def test_parts_of_heads(rot, norm):
    append((8, 2, 128), [3, 0], [411, 200], rot, norm=norm, fp8=norm, seed=rot)


def test_positions_strides_and_in_place():
    append((8, 2, 128), [9, 40], [350, 77], 128, positions=lambda p: (p * 7 + 3) % 513, stride_extra=264, in_place=True, seed=5)
    append((8, 8, 64), [9, 40], [350, 77], 64, True, positions=lambda p: p // 2, stride_extra=8, seed=6)


@pytest.mark.parametrize("heads", [(64, 8, 128), (72, 9, 128), (96, 12, 128), (160, 20, 128)])
def test_wide_tokens(heads):
    """Rings of four stages, and tokens of which four do not fit."""
    append(heads, [2, 0], [200, 150], 128, seed=7)


def test_pages_and_positions_outside_are_skipped_and_reported():
    import torch

    hq, hkv, d = 8, 2, 128
    prior, q_len = np.array([0, 30, 5], dtype=np.int32), np.array([200, 100, 220], dtype=np.int32)
    T = int(q_len.sum())
    c = Cache(hq, hkv, d, prior + q_len, seed=8)
    x = c.normal(T, hq + 2 * hkv, d)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    table = angles(230, d)
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(prior, q_len)]).astype(np.int32)
    outside = pos.copy()
    outside[[3, 299]] = [230, -1]
    bt = c.table.clone()
    bt[1, 4], bt[2, 2] = -1, 1 << 30
    bits = lambda r: [a.view(torch.int16).clone() for a in c.pa.gather(c.table[r], int(prior[r] + q_len[r]))]  # (a poisoned pool holds NaN)
    before = [bits(r) for r in range(3)]
    out = torch.full((T, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    c.pa.write_rope(q, k, v, bt, prior, q_len, table, positions=torch.from_numpy(outside).cuda(), q_out=out)
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_BOUNDS
    request = np.repeat(np.arange(3), q_len)
    bad = np.zeros(T, dtype=bool)
    bad[[3, 299]] = True
    bad |= (request == 1) & (pos // 16 == 4)
    bad |= (request == 2) & (pos // 16 == 2)
    bad = torch.from_numpy(bad).cuda()
    assert bool((out[bad] == 7.0).all())
    want, slack = turned(q, None, 0.0, table, torch.from_numpy(pos).cuda().long(), False)
    check_rounded(out[~bad], want[~bad], slack[~bad])
    t = 0
    for r, n in enumerate(q_len):
        gk, gv = bits(r)
        for i in range(int(n)):
            p = int(prior[r]) + i
            assert torch.equal(gv[p], before[r][1][p] if bool(bad[t]) else v[t].contiguous().view(torch.int16))
            if bool(bad[t]):
                assert torch.equal(gk[p], before[r][0][p])
            t += 1


def test_a_wait_that_runs_out_is_reported():
    import torch

    c, x, got = append((8, 2, 128), [9], [700], 128, seed=9)
    hq, hkv = 8, 2
    args = (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], c.table, [9], [700], angles(709, 128))
    want = c.pa.write_rope(*args)
    ps.ps_kv_set_wait_limit(c.pa.kv, 0)
    c.pa.write_rope(*args)
    with pytest.raises(ps.PsError) as e:
        c.pa.check_pool()
    assert e.value.status == ps.binding.PS_ERR_TIMEOUT
    ps.ps_kv_set_wait_limit(c.pa.kv, 2_000_000_000)
    again = c.pa.write_rope(*args)
    c.pa.check_pool()
    assert torch.equal(again, want)


def test_captured_and_replayed():
    import torch

    c, x, got = append((8, 2, 128), [9, 0], [500, 33], 128, seed=10)
    args = (x[:, :8].contiguous(), x[:, 8:10], x[:, 10:], c.table, [9, 0], [500, 33], angles(509, 128))
    want = c.pa.write_rope(*args)
    kv = [t[9:].clone() for t in c.pa.gather(c.table[0], 509)]  # (tokens 0 .. 8 were never written)
    out = torch.empty_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            c.pa.write_rope(*args, q_out=out)
            c.pa.write_rope(*args, q_out=out)
    c.pa.write_rope(args[0], args[2], args[1], *args[3:])  # other keys and values
    out.zero_()
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    assert all(torch.equal(a[9:], b) for a, b in zip(c.pa.gather(c.table[0], 509), kv))
    c.pa.check_pool()
