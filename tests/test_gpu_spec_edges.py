"""Calls of a speculative step at the edges of what their documentation allows."""
import glob
import os

import numpy as np
import pytest

import paper_2507_17769_b200 as ps
from paper_2507_17769_b200 import binding as B
from spec_util import Cache, tree_masks
from test_gpu_spec_cache import angles, append, check_fp8, check_rounded, turned

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def status_of(f):
    with pytest.raises(ps.PsError) as e:
        f()
    return e.value


@pytest.mark.parametrize("heads,fp8", [((8, 2, 128), False), ((8, 8, 64), False), ((8, 2, 128), True)])
@pytest.mark.parametrize("entry", [-1, -2, -3, -8, -(2 ** 31), 2 ** 31 - 1])
def test_every_page_outside_the_pool_is_reported(heads, fp8, entry):
    """... inside a sequence; entries behind its end are not looked at."""
    import torch

    prior, nodes = np.array([100, 30], dtype=np.int32), np.array([5, 2], dtype=np.int32)
    c = Cache(*heads, prior + nodes, seed=51, fp8=fp8).fill()
    mask, _ = tree_masks(nodes, 1, np.random.default_rng(1))
    q = c.normal(7, heads[0], heads[2])
    want = c.pa.run_tree(q, c.table, mask, prior, nodes)
    c.pa.check_pool()
    for page in (0, 3, 6):  # (the last holds drafted tokens)
        table = c.table.clone()
        table[0, page] = entry
        out, lse = c.pa.run_tree(q, table, mask, prior, nodes)
        assert status_of(c.pa.check_pool).status == B.PS_ERR_BOUNDS
        assert torch.equal(out[5:], want[0][5:]) and torch.equal(lse[5:], want[1][5:])
    table = c.table.clone()
    table[0, 7:], table[1, 2:] = entry, entry
    got = c.pa.run_tree(q, table, mask, prior, nodes)
    c.pa.check_pool()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("tokens", [1, 40, 296, 297, 900])
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 2, 64)])
def test_values_go_to_their_pages_bit_for_bit(tokens, heads):
    """A NaN's sign and payload too, with few tokens as with many, and as write() stores them."""
    import torch

    hq, hkv, d = heads
    c = Cache(hq, hkv, d, [tokens], seed=52)
    x = c.normal(tokens, hq + 2 * hkv, d)
    bits = x.view(torch.int16)
    for i, b in enumerate((0x7FC1, -0x3D, 0x7F81, -0x7F, 0x7F80, -0x80, -0x8000, 1)):
        bits[:, hq + hkv:, 3 + 7 * i] = b
    w = torch.ones(d, device="cuda", dtype=torch.bfloat16)
    v = x[:, hq + hkv:].contiguous()
    for cos_sin, weight in ((None, None), (angles(tokens, d), w)):
        c.pa.write_rope(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], c.table, [0], [tokens], cos_sin, q_weight=weight, k_weight=weight)
        for got in (c.pa.gather(c.table[0], tokens)[1], c.pa.read(c.table, [0], [tokens])[1]):
            assert torch.equal(got.view(torch.int16), v.view(torch.int16))
        c.pa.pool.fill_(0xFF)
    c.pa.write(x[:, hq:hq + hkv].contiguous(), v, c.table, [0], [tokens])
    assert torch.equal(c.pa.gather(c.table[0], tokens)[1].view(torch.int16), v.view(torch.int16))


def test_outputs_over_the_inputs_of_tree_attention_are_refused():
    """Results are stored while inputs are still read."""
    import torch

    prior, nodes = np.array([40], dtype=np.int32), np.array([9], dtype=np.int32)
    c = Cache(8, 2, 128, prior + nodes, seed=54).fill()
    mask, _ = tree_masks(nodes, 1, np.random.default_rng(1))
    room = c.normal(12, 8, 128)
    q = room[:9]
    want = c.pa.run_tree(q, c.table, mask, prior, nodes)
    floats = room.view(-1).view(torch.float32)

    def refused(**k):
        assert status_of(lambda: c.pa.run_tree(q, c.table, mask, prior, nodes, **k)).status == B.PS_ERR_INVALID

    before = room.clone()
    refused(out=q)
    refused(out=room[3:])
    refused(lse=floats[:72].view(9, 8))
    refused(lse=floats[9 * 512 - 8:9 * 512 + 64].view(9, 8))
    both = torch.empty(9 * 8 * 128 + 144, dtype=torch.bfloat16, device="cuda")
    refused(out=both[:9216].view(9, 8, 128), lse=both.view(torch.float32)[4600:4672].view(9, 8))
    long = torch.zeros(9 * 1024 // 4, dtype=torch.int64, device="cuda")
    long[2200:2209] = mask[:, 0]
    assert status_of(lambda: c.pa.run_tree(q, c.table, long[2200:2209].view(9, 1), prior, nodes, out=long.view(torch.bfloat16).view(9, 8, 128))).status == B.PS_ERR_INVALID
    assert torch.equal(room, before)
    got = c.pa.run_tree(q, c.table, mask, prior, nodes, out=both[:9216].view(9, 8, 128), lse=both.view(torch.float32)[4608:4680].view(9, 8))  # side by side
    c.pa.check_pool()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_what_went_wrong_is_named():
    """A wait that ran out in the append is told apart from one in tree attention, and a bounds error beside one is told too."""
    import torch

    c, x, _ = append((8, 2, 128), [9], [700], 128, seed=53)
    table = c.table.clone()
    table[0, 1] = -1

    def rope(bt=c.table):
        c.pa.write_rope(x[:, :8], x[:, 8:10], x[:, 10:], bt, [9], [700], angles(709, 128))

    def tree():
        c.pa.run_tree(x[:5, :8].contiguous(), c.table, torch.ones((5, 1), dtype=torch.int64, device="cuda"), [100], [5])

    def message(status):
        e = status_of(c.pa.check_pool)
        assert e.status == status
        c.pa.check_pool()  # the report is given once
        return str(e)

    rope(table)
    assert "outside the pool" in message(B.PS_ERR_BOUNDS)
    for calls, words, others in (((rope,), ("append",), ("attention", "outside the pool")), ((tree,), ("tree attention",), ("append", "outside the pool")),
                                 ((rope, tree), ("append", "tree attention"), ("outside the pool",))):
        for with_bounds in (False, True):
            if with_bounds:
                rope(table)
            ps.ps_kv_set_wait_limit(c.pa.kv, 0)
            for f in calls:
                f()
            torch.cuda.synchronize()
            ps.ps_kv_set_wait_limit(c.pa.kv, 2_000_000_000)
            text = message(B.PS_ERR_TIMEOUT)
            assert all(w in text for w in words), text
            assert all(w not in text for w in others if not (with_bounds and w == "outside the pool")), text
            assert ("outside the pool" in text) == with_bounds, text


def test_the_documented_step():
    """The example of a speculative step in the documentation, as it stands there: drafted tokens are rotated by their positions in their sequences."""
    import torch

    (path,) = glob.glob(os.path.join(ROOT, "READ*"))
    blocks = open(path).read().split("```python\n")[1:]
    code = [b.split("```")[0] for b in blocks if "write_rope(" in b]
    assert len(code) == 1
    prior, n_nodes = np.array([50, 0, 7], dtype=np.int32), np.array([9, 1, 20], dtype=np.int32)
    pa_cache = Cache(8, 2, 128, prior + n_nodes, seed=55).fill()
    mask, sees = tree_masks(n_nodes, 1, np.random.default_rng(2))
    depth = np.concatenate([s.sum(1) - 1 for s in sees]).astype(np.int32)
    x = pa_cache.normal(30, 12, 128)
    qw, kw = ((1 + 0.3 * torch.randn(128, generator=pa_cache.gen, device="cuda")).bfloat16() for _ in range(2))
    table = angles(64, 128)
    names = dict(pa=pa_cache.pa, q=x[:, :8], k_new=x[:, 8:10], v_new=x[:, 10:], block_table=pa_cache.table, prior=prior, n_nodes=n_nodes, cos_sin=table,
                 depth=torch.from_numpy(depth).cuda(), qw=qw, kw=kw, mask=mask, index=torch.zeros((3, 1), dtype=torch.int32, device="cuda"),
                 count=torch.ones(3, dtype=torch.int32, device="cuda"), begin=prior, length=n_nodes, np=np, torch=torch)
    exec(compile(code[0], "example", "exec"), names)
    pa_cache.pa.check_pool()
    pos = torch.from_numpy(np.repeat(prior, n_nodes) + depth).cuda().long()
    check_rounded(names["q"], *turned(x[:, :8], qw, 1e-6, table, pos, False))
    check_rounded(names["k"], *turned(x[:, 8:10], kw, 1e-6, table, pos, False))
    assert torch.equal(names["v"], x[:, 10:])


def test_positions_beyond_32_bits_are_refused():
    """... by every call, however wide the block table: kernels count them in 32 bits."""
    import torch

    pa = ps.PagedAttention(8, 2, 128, 8)
    x = torch.zeros((512, 12, 128), dtype=torch.bfloat16, device="cuda")
    some = torch.zeros(1 << 16, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.ps_attn_tree_workspace(pa.shape) + 256, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) // 256 * 256
    q, out = (torch.zeros((256, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k = torch.zeros((256, 2, 128), dtype=torch.bfloat16, device="cuda")
    rope = B.ps_rope(q_dev=x.data_ptr(), k_new_dev=x.data_ptr() + 2048, v_new_dev=x.data_ptr() + 2560, q_out_dev=out.data_ptr(), q_stride=1536, k_stride=1536, v_stride=1536)
    pages = 2 ** 27 + 32  # 2^31 + 512 tokens
    calls = {"write": lambda a, b: B.ps_kv_write(pa.kv, k, k, some, pages, a, b), "write_rope": lambda a, b: B.ps_kv_write_rope(pa.kv, rope, some, pages, a, b),
             "run_tree": lambda a, b: B.ps_attn_tree(pa.kv, q, some, pages, some, 4, a, b, out, None, at, ws.numel() - 256),
             "accept": lambda a, b: B.ps_kv_accept(pa.kv, some, pages, a, b, some, 4, some), "read": lambda a, b: B.ps_kv_read(pa.kv, some, pages, a, b, k, k),
             "plan": lambda a, b: B.ps_attn_plan(pa.shape, a, b, pages)}
    for name, call in calls.items():
        for prior, length in ((2 ** 31 - 8, 16), (2 ** 31 - 1, 1), (2 ** 31 - 200, 200), (2 ** 31 - 256, 1)):
            e = status_of(lambda: call([prior], [length]))
            assert e.status == B.PS_ERR_INVALID and "more than" in str(e), (name, prior, length, str(e))
    pa.check_pool()


def test_lengths_are_refused_before_results_are_allocated():
    """2^31 - 1 tokens a request would be half a terabyte of K."""
    import torch

    pa = ps.PagedAttention(8, 2, 128, 4)
    table = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    for length in ([2 ** 31 - 1, 1], [2 ** 31 - 1, 2 ** 31 - 1], [65, 0], [2 ** 31 - 1, -1]):
        assert status_of(lambda: pa.read(table, [0, 0], length)).status == B.PS_ERR_INVALID


def test_outputs_over_the_inputs_of_the_cache_calls_are_refused():
    """What a call reads for other tokens must not change while one token's results are stored."""
    import torch

    c = Cache(2, 1, 64, [32], seed=56).fill()
    x = c.normal(32, 4, 64)
    room = torch.zeros(3 * 32 * 128, dtype=torch.bfloat16, device="cuda")
    out = room[4096:8192].view(32, 2, 64)
    w, cs, pos = torch.ones(64, dtype=torch.bfloat16, device="cuda"), angles(32, 64), torch.arange(32, dtype=torch.int32, device="cuda")
    good = dict(cos_sin=cs, positions=pos, q_weight=w, k_weight=w, block_table_dev=c.table)
    inside = {"cos_sin": room[1024:5120].view(torch.float32).view(32, 64), "positions": room[8000:8064].view(torch.int32), "q_weight": room[8176:8240], "k_weight": room[4040:4104],
              "block_table_dev": room[4092:4092 + 2 * c.table.numel()].view(torch.int32).view(c.table.shape)}

    def call(**k):
        k = {**good, **k}
        return c.pa.write_rope(x[:, :2], x[:, 2:3], x[:, 3:], k.pop("block_table_dev"), [0], [32], q_out=out, **k)

    for name, t in inside.items():
        t.copy_(good[name])
        assert status_of(lambda: call(**{name: t})).status == B.PS_ERR_INVALID, name
    beside = {"cos_sin": room[:4096].view(torch.float32).view(32, 64), "positions": room[8192:8256].view(torch.int32), "q_weight": room[8256:8320], "k_weight": room[8320:8384],
              "block_table_dev": room[8384:8384 + 2 * c.table.numel()].view(torch.int32).view(c.table.shape)}
    want = c.pa.write_rope(x[:, :2], x[:, 2:3], x[:, 3:], c.table, [0], [32], cs, positions=pos, q_weight=w, k_weight=w)
    for name, t in beside.items():
        t.copy_(good[name])
    assert torch.equal(call(**beside), want)
    k, v = (torch.empty(32, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = beside["block_table_dev"]
    over = room[8320:8320 + 2048]
    for a, b, bt in ((k, k, c.table), (over, v, table), (k, over, table), (None, over, table), (room[:2048], room[2040:4088], c.table)):
        assert status_of(lambda: B.ps_kv_read(c.pa.kv, bt, bt.size(1), [0], [32], a, b)).status == B.PS_ERR_INVALID
    B.ps_kv_read(c.pa.kv, table, table.size(1), [0], [32], room[:2048], room[2048:4096])
    c.pa.check_pool()
    assert torch.equal(room[:2048].view(32, 1, 64), c.pa.read(c.table, [0], [32])[0]) and torch.equal(room[2048:4096].view(32, 1, 64), x[:, 3:])


@pytest.mark.parametrize("heads,fp8", [((2, 1, 64), False), ((2, 2, 128), True)])
def test_paths_and_stretches_of_more_requests_than_a_launch_takes(heads, fp8):
    import torch

    n = 8100
    rng = np.random.default_rng(57)
    prior, nodes = rng.integers(0, 20, n).astype(np.int32), rng.integers(1, 6, n).astype(np.int32)
    c = Cache(*heads, prior + nodes, seed=58, fp8=fp8).fill()
    index = np.full((n, 3), -7, dtype=np.int32)
    count = np.minimum(rng.integers(0, 4, n), nodes).astype(np.int32)
    for r in range(n):
        index[r, :count[r]] = np.sort(rng.choice(nodes[r], count[r], replace=False))
    start = np.cumsum(prior + nodes) - prior - nodes
    source = np.arange(int((prior + nodes).sum()))
    for r in range(n):
        at = start[r] + prior[r]
        source[at:at + count[r]] = at + index[r, :count[r]]
    before = c.pa.read(c.table, np.zeros(n, dtype=np.int32), prior + nodes)
    c.pa.accept(c.table, prior, nodes, torch.from_numpy(index).cuda(), torch.from_numpy(count).cuda())
    after = c.pa.read(c.table, np.zeros(n, dtype=np.int32), prior + nodes)
    c.pa.check_pool()
    assert torch.equal(before[0], torch.cat(c.k).bfloat16()) and torch.equal(before[1], torch.cat(c.v).bfloat16())
    assert all(torch.equal(b, a[torch.from_numpy(source).cuda()]) for a, b in zip(before, after))


@pytest.mark.parametrize("tokens", [40, 700])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("which", ["q", "k"])
@pytest.mark.parametrize("fp8", [False, True])
def test_a_norm_of_queries_or_of_keys_alone(tokens, interleaved, which, fp8):
    import torch

    c = Cache(8, 2, 128, [tokens], seed=59, fp8=fp8)
    x = c.normal(tokens, 12, 128, scale=3.0)
    w = (1 + 0.3 * torch.randn(128, generator=c.gen, device="cuda")).bfloat16()
    weight = {"q": None, "k": None, which: w}
    table = angles(tokens, 96)
    q = c.pa.write_rope(x[:, :8], x[:, 8:10], x[:, 10:], c.table, [0], [tokens], table, q_weight=weight["q"], k_weight=weight["k"], interleaved=interleaved)
    c.pa.check_pool()
    pos = torch.arange(tokens, device="cuda")
    check_rounded(q, *turned(x[:, :8], weight["q"], 1e-6, table, pos, interleaved))
    want, slack = turned(x[:, 8:10], weight["k"], 1e-6, table, pos, interleaved)
    if fp8:
        kc, _, ks, _ = c.pa.gather_fp8(c.table[0], tokens)
        check_fp8(kc, ks, want, slack)
    else:
        check_rounded(c.pa.gather(c.table[0], tokens)[0], want, slack)
