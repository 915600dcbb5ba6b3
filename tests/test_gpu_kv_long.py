"""Attention with rows in blocks of several eights over units long enough for a warp's ring to go round, for its page table to be looked
up again (after 32 tiles of its own), and for many CTAs to have parts of a unit.  Oracle and tolerances of test_gpu_kv.py."""
import pytest
import torch

from oracle import kv as O
from test_gpu_kv import DEV, attend, close, ints, on_device, pool
from test_gpu_kv_ranges import eights_per_block

pytestmark = pytest.mark.gpu
WIDE = 2500              # pages of 64 behind a table's own: more than 16 chunks per SM, so that rows come in blocks of several eights


@pytest.mark.parametrize("Q,group,D,eights", [(2, 8, 64, 2), (5, 4, 64, 3), (4, 8, 64, 4), (5, 8, 64, 3), (2, 8, 128, 2), (5, 4, 128, 3), (4, 8, 128, 4),
                                              (5, 8, 128, 3), (2, 8, 256, 2), (4, 8, 256, 2), (5, 8, 256, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_long_units_of_several_eights(ears, dtype, Q, group, D, eights):
    for H, lengths in ((1, [12001]), (2, [7000, 3])):
        wide = WIDE * 64 + max(lengths)
        assert eights_per_block(ears, D, H, len(lengths), Q, group, wide) == eights
        attend(ears, dtype, lengths, Q, group, H, D, 64, seed=D + Q, table_extra=WIDE, sharp=2.0)


@pytest.mark.parametrize("Q,group,D", [(2, 8, 64), (4, 8, 64), (5, 4, 128), (4, 8, 128), (2, 8, 256)])
def test_whole_units_of_several_eights(ears, Q, group, D):
    """As many sequences as fill the GPU, each longer than 32 tiles per warp, pages shared: units that one CTA has whole."""
    codes, params, pages, g = pool([2700], 2, D, 16, D)
    copies = 200
    q = torch.randn(1, Q, 2 * group, D, generator=g).bfloat16()
    want = O.attention(q, codes, params, pages, [2700 - Q])
    got, lse = ears.kv_attention(q.to(DEV).expand(copies, -1, -1, -1), on_device(ears, codes, params), pages.to(DEV).expand(copies, -1),
                                 ints([2700 - Q] * copies), lse=True)
    for b in (0, 1, 99, 198, 199):
        close(got[b:b + 1], want, "bf16", lse[b:b + 1])
    spread = (got.float() - got[:1].float()).abs().amax()          # the order of sums differs with where CTAs begin
    assert spread <= 2.0 ** -6 * got.float().abs().amax()


@pytest.mark.parametrize("Q,group,D", [(4, 4, 64), (5, 4, 128), (2, 8, 256)])
def test_sizes_that_differ_widely_in_blocks_of_several_eights(ears, Q, group, D):
    codes, params, pages, g = pool([3000], 2, D, 16, 21)
    row = torch.randint(-30, 31, (codes.shape[0], 1, 2, 16, 1, 1), generator=g).double()
    params[:, 1:] = (params[:, 1:].double() * 2.0 ** row).bfloat16()
    params[:, :1] = (params[:, :1].double() * 2.0 ** -40).bfloat16()
    q = torch.randn(1, Q, 2 * group, D, generator=g)
    q[0, 0] *= 2.0 ** -20
    q[0, -1] *= 8.0
    q = (q * 2.0 ** 40).bfloat16()
    want = O.attention(q, codes, params, pages, [3000 - Q])
    table = torch.nn.functional.pad(pages, (0, 4 * WIDE), value=-1).to(DEV)
    got, lse = ears.kv_attention(q.to(DEV), on_device(ears, codes, params), table, ints([3000 - Q]), lse=True)
    close(got, want, "bf16", lse)


def test_sequences_that_are_left_out_wherever_they_stand(ears):
    """A padded batch: positions of no meaning are not formed, reported or waited for."""
    codes, params, pages, g = pool([50] * 4, 2, 64, 16, 33)
    start, counts = [2**31 - 1, 47, -2**31, 2**31 - 2], [0, 3, 0, 0]
    q, status = torch.randn(4, 3, 4, 64, generator=g).half().to(DEV), ints([0])
    for window, sinks in ((0, 0), (2**31 - 1, 2**31 - 1), (5, 3)):
        out, lse = ears.kv_attention(q, on_device(ears, codes, params), pages.to(DEV), ints(start), ints(counts), window=window, sinks=sinks, lse=True,
                                     status=status)
        close(out[1:2], O.attention(q[1:2].cpu(), codes, params, pages[1:2], [47], window=window, sinks=sinks), "fp16", lse[1:2])
        for b in (0, 2, 3):
            assert not out[b].any() and (lse[b] == -torch.inf).all()
    cache = on_device(ears, codes, params)
    x = torch.randn(4, 3, 2, 64, device=DEV)
    ears.kv_write(cache, x, x, pages.to(DEV), ints(start), ints([0] * 4), status=status)
    k, v = ears.kv_read(cache, pages.to(DEV), ints(start), 3, ints([0] * 4), status=status)
    assert status.item() == 0 and not k.any() and not v.any()
    assert torch.equal(cache.codes.cpu(), codes) and torch.equal(cache.params.cpu(), params)
