"""Prefills over 8-bit codes whose keys the call would turn once, into a copy: in a workspace that ends where the copy would
begin they turn in the attention kernel, and give the same within what that rounds."""
import pytest
import torch

from tests import test_gpu_kv8 as kv8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("case", range(len(kv8.COPIED)))
def test_without_room_for_the_copy(case):
    hq, hkv, d, lens, tile, split = kv8.COPIED[case]
    b = kv8.Batch(lens, hq, hkv, d, torch.bfloat16, kv8.CODES[case // 2 % 2], style=case % 2, seed=case + 20)
    extra = kv8.copied_bytes(b)
    assert extra > 0 and kv8.tile_of(b) == (tile, split)
    room = b.ws.numel() - extra
    ws = torch.full((room + extra,), 0xa5, dtype=torch.uint8, device="cuda")
    got = b.run(ws=ws[:max(1, room)])
    b.check(got, f"case {case}")
    # one byte less than the copy needs is as good as none
    assert torch.equal(b.run(ws=ws[:room + extra - 1]), got)
    assert (ws[max(1, room):] == 0xa5).all()
