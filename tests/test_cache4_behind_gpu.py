"""Calls on the 4-bit cache one right behind the other, each reading what the one before has just written: queries, lengths, weights, slots, tables.
Kernels start while the one before them drains; with and without waiting for each call the results are the same."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    yield attention
    attention.device_status()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("batch,tokens,context", [(1, 1, 3000), (40, 1, 500), (3, 7, 900), (2, 160, 2600)])
def test_each_call_reads_what_the_one_before_wrote(A, dtype, batch, tokens, context):
    """Over and over in the same tensors: rotated queries from the append to the attention, received weight on to the eviction, its lengths and weights to another
    attention; between the rounds slots, lengths, offsets, positions and tables are overwritten in place, right before they are used."""
    hkv, group, d, page, budget, rounds = 2, 4, 128, 16, 200, 10
    width, out_width = -(-context // page), -(-(budget + tokens) // page)
    pages = batch * (width + out_width)
    g = torch.Generator(device="cuda")
    g.manual_seed(batch + tokens)
    T = batch * tokens
    fill = torch.randn(2, pages * page, hkv, d, device="cuda", generator=g).to(dtype)
    x = torch.randn(rounds, T, (group + 2) * hkv, d, device="cuda", generator=g).to(dtype)
    angle = torch.rand(context, d // 2, device="cuda", generator=g) * 6
    cos, sin = angle.cos(), angle.sin()
    plans = []
    for _ in range(rounds):
        perm = torch.randperm(pages, device="cuda", generator=g)
        table, out_table = perm[:batch * width].view(batch, width), perm[batch * width:].view(batch, out_width)
        lens = torch.randint(tokens, context + 1, (batch,), device="cuda", generator=g)
        place = lens[:, None] - tokens + torch.arange(tokens, device="cuda")
        slots = (table.gather(1, place // page) * page + place % page).flatten()
        plans.append((slots, place.flatten().int(), table.int(), out_table.int(), lens.int()))
    starts = (torch.arange(batch + 1, device="cuda") * tokens).int()

    def run(wait):
        cache = A.cache4(pages, hkv, page, d)
        A.kv_append4(fill[0], fill[1], cache, torch.arange(pages * page, device="cuda"))
        q, fresh, seen = torch.empty(T, hkv * group, d, dtype=dtype, device="cuda"), torch.empty_like(x[0]), []
        weights = torch.zeros(batch, hkv, width * page, device="cuda")
        slots, positions, table, out_table, lens = (t.clone() for t in plans[0])
        torch.cuda.synchronize()
        for i in range(rounds):
            fresh.copy_(x[i])
            for to, new in zip((slots, positions, table, out_table, lens), plans[i]):
                to.copy_(new)
            wait()
            xq, k, v = fresh.split([group * hkv, hkv, hkv], 1)
            A.kv_append4(k, v, cache, slots, positions=positions, cos=cos, sin=sin, q=xq, q_out=q)
            wait()
            out, _ = A.paged_attention4(q, cache, table, lens, q_start=starts, max_q_len=tokens, weights=weights, weights_out=weights)
            wait()
            left, kept, moved = A.kv_evict4(cache, table, lens, weights, out_table, budget, 2, 9)
            wait()
            A.kv_append4(k, v, cache, slots, positions=positions, cos=cos, sin=sin, q=q, q_out=q)       # turned once more, in place
            wait()
            after, more = A.paged_attention4(q[:batch], cache, out_table, left, weights=moved)
            wait()
            rows, _ = A.kv_read4(cache, slots, dtype)
            seen += [out, left, kept, moved, after, more, rows, q.clone(), weights.clone()]
            wait()
        torch.cuda.synchronize()
        return seen

    patient = run(torch.cuda.synchronize)
    assert all(torch.isfinite(t).all() for t in patient)
    for _ in range(4):
        for a, b in zip(run(lambda: None), patient):
            assert torch.equal(a, b)
    A.device_status()
