"""What the calls of a speculative step refuse before they reach the device."""
import numpy as np
import pytest
import torch

import paper_2507_17769_b200 as ps
from paper_2507_17769_b200 import binding as B
from test_tensor_calls_host import host_session

BF, I32, I64, F32 = torch.bfloat16, torch.int32, torch.int64, torch.float32
HQ, HKV, D, T = 8, 2, 64, 5  # as in host_session


def session():
    return host_session()


def args(call):
    table = torch.zeros((2, 4), dtype=I32)
    if call == "write_rope":
        return dict(q=torch.zeros((T, HQ, D), dtype=BF), k_new=torch.zeros((T, HKV, D), dtype=BF), v_new=torch.zeros((T, HKV, D), dtype=BF), block_table_dev=table,
                    prior=[0, 3], q_len=[2, 3], cos_sin=torch.zeros((9, 32)), positions=torch.zeros(T, dtype=I32), q_weight=torch.zeros(D, dtype=BF),
                    k_weight=torch.zeros(D, dtype=BF), q_out=torch.zeros((T, HQ, D), dtype=BF))
    if call == "run_tree":
        return dict(q=torch.zeros((T, HQ, D), dtype=BF), block_table_dev=table, mask=torch.zeros((T, 1), dtype=I64), prior=[0, 3], n_nodes=[2, 3],
                    out=torch.zeros((T, HQ, D), dtype=BF), lse=torch.zeros((T, HQ)))
    if call == "accept":
        return dict(block_table_dev=table, prior=[0, 3], n_nodes=[2, 3], index=torch.zeros((2, 3), dtype=I32), count=torch.zeros(2, dtype=I32))
    return dict(block_table_dev=table, begin=[0, 3], length=[2, 3])


CALLS = ["write_rope", "run_tree", "accept", "read"]


@pytest.mark.parametrize("call", CALLS)
def test_good_tensors_come_as_far_as_the_null_pool(call):
    with pytest.raises(ps.PsError) as e:
        getattr(session(), call)(**args(call))
    assert e.value.status == B.PS_ERR_INVALID


def strided(x):
    return torch.stack([x, x], dim=-1)[..., 0]


TENSORS = [(c, n) for c in CALLS for n, x in args(c).items() if isinstance(x, torch.Tensor)]


@pytest.mark.parametrize("call,name", TENSORS)
def test_other_types_extents_and_layouts_are_refused(call, name):
    x = args(call)[name]
    wrong = [x.double(), x[..., None], strided(x), x.to("meta")]
    if name not in ("block_table_dev", "cos_sin"):
        wrong += [x[:-1]]
    if name == "block_table_dev":
        wrong += [x[:1]]
    if x.dim() == 3:
        wrong += [x[:, 1:], x[..., : D // 2], torch.zeros_like(x).transpose(0, 1)]
    for y in wrong:
        with pytest.raises(AssertionError):
            getattr(session(), call)(**{**args(call), name: y})
    with pytest.raises(TypeError):
        getattr(session(), call)(**{**args(call), name: "x"})


def test_slices_of_one_projection_are_taken_and_broadcast_tokens_are_not():
    x = torch.zeros((T, HQ + 2 * HKV, D), dtype=BF)
    a = {**args("write_rope"), "q": x[:, :HQ], "k_new": x[:, HQ:HQ + HKV], "v_new": x[:, HQ + HKV:]}
    with pytest.raises(ps.PsError):
        session().write_rope(**a)
    for name in ("q", "k_new", "v_new"):
        with pytest.raises(AssertionError):
            session().write_rope(**{**a, name: a[name][:1].expand(T, -1, -1)})


@pytest.mark.parametrize("call", CALLS)
def test_lengths_that_do_not_belong_together(call):
    first, second = ("begin", "length") if call == "read" else ("prior", "q_len" if call == "write_rope" else "n_nodes")
    for a, b in (([0], [2, 3]), ([0, 3], [5]), ([[0, 3]], [[2, 3]])):
        with pytest.raises(ValueError):
            getattr(session(), call)(**{**args(call), first: a, second: b})
    if call in ("write_rope", "run_tree"):
        with pytest.raises(AssertionError):  # (they say how many tokens there are)
            getattr(session(), call)(**{**args(call), second: [2, 2]})


def test_null_arguments_through_addresses():
    z = np.zeros(1, dtype=np.int32)
    for f in (lambda: B.ps_kv_write_rope(None, B.ps_rope(), 1, 1, z, z + 1), lambda: B.ps_attn_tree(None, 16, 16, 1, 16, 1, z, z + 1, 16, None, 256, 0),
              lambda: B.ps_kv_accept(None, 16, 1, z, z + 1, 16, 1, 16), lambda: B.ps_kv_read(None, 16, 1, z, z + 1, 16, 16), lambda: B.ps_kv_set_wait_limit(None, 1)):
        with pytest.raises(ps.PsError) as e:
            f()
        assert e.value.status == B.PS_ERR_INVALID
    with pytest.raises(ValueError):
        B.ps_kv_read(None, 16, 1, z, np.ones(2, dtype=np.int32), 16, 16)


def test_the_workspace_depends_on_the_shape_alone():
    big, small = (B.ps_attn_tree_workspace(ps.make_shape(32, 8, d)) for d in (128, 64))
    assert big > small > 0 and big % 256 == 0
    assert B.ps_attn_tree_workspace(ps.make_shape(8, 8, 128)) == big
    with pytest.raises(ps.PsError):
        B.ps_attn_tree_workspace(ps.make_shape(32, 8, 96))


@pytest.mark.gpu
def test_refusals_of_the_library():
    pa = ps.PagedAttention(HQ, HKV, D, 8)
    x = torch.zeros((64, HQ + 2 * HKV, D), dtype=BF, device="cuda")
    table = torch.zeros((2, 4), dtype=I32, device="cuda")
    cs = torch.zeros((9, 64), device="cuda")

    def refused(status, f, *a, **k):
        with pytest.raises(ps.PsError) as e:
            f(*a, **k)
        assert e.value.status == status, e.value
        assert ps.ps_last_error()

    def rope(prior, q_len, cos_sin=cs, **k):
        n = sum(q_len)
        return pa.write_rope(x[:n, :HQ], x[:n, HQ:HQ + HKV], x[:n, HQ + HKV:], table, prior, q_len, cos_sin, **k)

    def tree(prior, nodes, words=1):
        n = sum(nodes)
        return pa.run_tree(torch.zeros((n, HQ, D), dtype=BF, device="cuda"), table, torch.zeros((n, words), dtype=I64, device="cuda"), prior, nodes)

    inv, uns = B.PS_ERR_INVALID, B.PS_ERR_UNSUPPORTED
    refused(inv, rope, [62, 0], [3, 1])          # beyond the table's pages
    refused(inv, rope, [-1, 0], [3, 1])
    refused(inv, rope, [0, 0], [3, 0])
    refused(uns, rope, [0, 0], [3, 1], cos_sin=cs[:, :40].contiguous())
    refused(uns, rope, [0, 0], [3, 1], cos_sin=torch.zeros((9, 80), device="cuda"))
    refused(inv, rope, [0, 0], [3, 1], cos_sin=torch.zeros((0, 64), device="cuda"))
    refused(inv, rope, [0, 0], [3, 1], eps=-1.0)
    refused(inv, rope, [0, 0], [3, 1], eps=float("nan"))
    flat = x.view(-1)
    odd = flat[4:4 + 4 * HQ * D].view(4, HQ, D)  # 8 bytes off
    refused(inv, pa.write_rope, odd, x[:4, :HKV].contiguous(), x[:4, :HKV].contiguous(), table, [0, 0], [3, 1], cs)
    wide = flat[:4 * (HQ * D + 4)].view(4, HQ * D + 4)[:, :HQ * D].unflatten(1, (HQ, D))
    refused(inv, pa.write_rope, wide, x[:4, :HKV].contiguous(), x[:4, :HKV].contiguous(), table, [0, 0], [3, 1], cs)
    n = 4 * HQ * D
    for shift in (0, 8, HQ * D):  # q_out over the projection's own rows
        refused(inv, rope, [0, 0], [3, 1], q_out=flat[shift:shift + n].view(4, HQ, D))
    refused(inv, tree, [62, 0], [3, 1])
    refused(inv, tree, [0, 0], [65 - 1, 0])
    refused(inv, tree, [-1, 0], [3, 1])
    refused(uns, tree, [0, 0], [3, 1], 5)
    refused(inv, tree, [0, 0], [3, 1], 0)  # (an empty tensor has no address)
    long = torch.zeros((1, 20), dtype=I32, device="cuda")
    refused(inv, pa.run_tree, torch.zeros((65, HQ, D), dtype=BF, device="cuda"), long, torch.zeros((65, 1), dtype=I64, device="cuda"), [0], [65])
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    q = torch.zeros((1, HQ, D), dtype=BF, device="cuda")
    refused(B.PS_ERR_WORKSPACE, B.ps_attn_tree, pa.kv, q, table, 4, torch.zeros(1, dtype=I64, device="cuda"), 1, [0], [1], q, None, ws, 1 << 20)
    index, count = torch.zeros((2, 3), dtype=I32, device="cuda"), torch.zeros(2, dtype=I32, device="cuda")
    refused(inv, pa.accept, table, [0, 62], [1, 3], index, count)
    refused(inv, pa.accept, table, [0, 0], [1, 0], index, count)
    refused(inv, pa.accept, table, [0, 0], [1, 1], index[:, :0].contiguous(), count)
    refused(inv, pa.read, table, [0, -1], [1, 1])
    refused(inv, pa.read, table, [0, 0], [1, -1])
    refused(inv, pa.read, table, [0, 63], [1, 2])
    refused(inv, ps.ps_kv_set_wait_limit, pa.kv, -1)
    refused(inv, ps.ps_kv_set_wait_limit, pa.kv, 5_000_000_000)
    pa.check_pool()
    pa.close()
    for f in (lambda: rope([0, 0], [3, 1]), lambda: tree([0, 0], [3, 1]), lambda: pa.accept(table, [0, 0], [1, 1], index, count), lambda: pa.read(table, [0, 0], [1, 1])):
        refused(inv, f)
