"""Calls with the widest tables that the 4-bit cache takes: counts and offsets that come near 31 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE = 128
WIDEST = 0x7fffff00


@pytest.fixture(scope="module")
def A():
    from paper_2603_08343_b200 import build
    build.build()
    from paper_2603_08343_b200 import attention
    yield attention
    attention.device_status()


def filled(A, pages, hkv, page, d, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    cache = A.cache4(pages, hkv, page, d)
    k, v = (torch.randn(pages * page, hkv, d, device="cuda", generator=g) for _ in range(2))
    A.kv_append4(k, v, cache, torch.arange(pages * page, device="cuda"))
    return cache, g


@pytest.mark.parametrize("group", [16, 1])                            # more rows than scores are kept for; more scores than there is room for
@pytest.mark.parametrize("keys", [WIDEST, WIDEST - PAGE])             # the last chunk of 512 keys ends past 2^31 - 1, whole and cut
def test_received_weight_of_the_widest_tables(A, keys, group):
    cache, g = filled(A, 8, 1, PAGE, 64)
    width, n = keys // PAGE, 700
    table = torch.full((1, width), 1 << 30, dtype=torch.int32, device="cuda")     # no page: what is looked at behind the length is reported
    table[0, :6] = torch.arange(6, dtype=torch.int32, device="cuda")
    q = torch.randn(1, group, 64, device="cuda", generator=g).bfloat16()
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    narrow, want = A.paged_attention4(q, cache, table[:, :6].contiguous(), lens, weights_out=torch.empty(1, 1, 6 * PAGE, device="cuda"))
    received = torch.ones(1, 1, keys, device="cuda")
    out, received = A.paged_attention4(q, cache, table, lens, weights_out=received)
    A.device_status()
    assert (out - narrow).abs().max() <= 2.0 ** -7 * narrow.abs().max()
    assert ((received[0, 0, :n] - want[0, 0, :n]).abs() <= 1e-5 * want[0, 0, :n] + 1e-12).all()
    assert not received[0, 0, n:].any()


def test_received_weight_of_no_tokens_over_the_widest_table(A):
    cache, _ = filled(A, 1, 1, PAGE, 64)
    received = torch.ones(1, 1, WIDEST, device="cuda")
    A.paged_attention4(torch.empty(0, 4, 64, device="cuda"), cache, torch.zeros(1, WIDEST // PAGE, dtype=torch.int32, device="cuda"),
                       torch.tensor([5], dtype=torch.int32, device="cuda"), q_start=torch.zeros(2, dtype=torch.int32, device="cuda"),
                       weights=received, weights_out=received)
    A.device_status()
    assert (received[0, 0, :5] == 1).all() and not received[0, 0, 5:].any()


def test_received_weight_of_as_many_keys_as_there_can_be(A):
    """Each of 2^31 - 256 keys (the same few pages over and over) receives its part of nine rows."""
    cache, g = filled(A, 8, 1, PAGE, 64)
    width = WIDEST // PAGE
    table = torch.arange(width, dtype=torch.int32, device="cuda").remainder_(8)[None]
    q = torch.randn(1, 9, 64, device="cuda", generator=g).bfloat16()
    out, received = A.paged_attention4(q, cache, table, torch.tensor([WIDEST], dtype=torch.int32, device="cuda"),
                                       weights_out=torch.empty(1, 1, WIDEST, device="cuda"))
    A.device_status()
    once, _ = A.paged_attention4(q, cache, table[:, :8].contiguous(), torch.tensor([8 * PAGE], dtype=torch.int32, device="cuda"),
                                 weights_out=torch.empty(1, 1, 8 * PAGE, device="cuda"))
    assert (out - once).abs().max() <= 2.0 ** -6 * once.abs().max()
    whole = received[0, 0, :width // 8 * 8 * PAGE].view(-1, 8 * PAGE)
    assert (whole == whole[0]).all()                                   # a key's weight does not depend on where it lies
    assert abs(received.sum(dtype=torch.float64).item() - 9) <= 1e-3
