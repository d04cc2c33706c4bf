"""What slope_gated_fwd_workspace_bytes answers is enough for every call that its arguments describe: with the adapter of that rank or, L and R
both NULL, without one, and for h alone where something may be kept."""
import random

import pytest
import torch

from paper_2405_16325_amd import binding as sl

# the product without an adapter is split into more slabs than the one with it
MORE_WITHOUT = [(51, 7104, 4736, 32), (80, 12032, 18432, 32), (97, 9280, 2384, 32), (47, 5568, 6048, 32), (47, 5568, 6048, 128), (37, 8128, 10584, 32)]


def drawn():
    rng = random.Random(3)
    return [(int(2 ** rng.uniform(0, 14)), 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 12)), rng.choice([32, 64, 128, 512])) for _ in range(20000)]


def test_room_for_an_adapter_is_room_without_one():
    size = sl.lib().slope_gated_fwd_workspace_bytes
    for b, d_in, d_ff, r in MORE_WITHOUT + drawn():
        for kept in (0, 8, 16):
            assert size(b, d_in, d_ff, r, kept) >= size(b, d_in, d_ff, 0, kept) >= size(b, d_in, d_ff, 0, 0), (b, d_in, d_ff, r, kept)


@pytest.mark.gpu
@pytest.mark.parametrize("b,d_in,d_ff,r", MORE_WITHOUT[:1] + MORE_WITHOUT[2:5])
def test_a_buffer_of_that_size_is_taken(b, d_in, d_ff, r):
    print(f"gated_fwd without an adapter in room for rank {r}: b={b} d_ff={d_ff} d_in={d_in}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(b)
    x = torch.randn(b, d_in, generator=gen, device="cuda").to(sl.BF16)
    vals, meta, _ = sl.slope_prune_rows(torch.randn(2 * d_ff, d_in, generator=gen, device="cuda").mul_(d_in ** -0.5).to(sl.BF16))
    want = sl.slope_gated_fwd(x, vals, meta)[0]
    need = sl.lib().slope_gated_fwd_workspace_bytes(b, d_in, d_ff, r, 0)
    whole = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    h = torch.empty_like(want)
    status = sl.lib().slope_gated_fwd(x.data_ptr(), b, vals.data_ptr(), meta.data_ptr(), d_ff, d_in, sl.SLOPE_ACT_SILU, None, None, r, h.data_ptr(), None,
                                      None, None, whole.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == sl.SLOPE_OK and torch.equal(h, want) and (whole[need:] == 7).all()
