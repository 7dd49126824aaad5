"""-m gpu: opt_tree_kv_compact against a plain 64-bit form (exact)."""
import numpy as np
import pytest
import torch

from paper_2406_17276_b200 import binding
from tests import _kv

pytestmark = pytest.mark.gpu


def _paths(rs, nodes, keep, G):
    gather = np.full((len(nodes), G), -1, np.int32)
    for b, (x, m) in enumerate(zip(nodes, keep)):
        if m:
            gather[b, :m] = np.concatenate([[0], 1 + np.sort(rs.choice(x, m - 1, replace=False))]) if x else [0]
    return gather


def _run(case, keep, G, scales=(-8, -5), gather=None):
    kv = case.handle(binding)
    tensors = case.cache(scales=scales)
    cache = binding.KVCache(*tensors)
    gather = _paths(case.rs, case.step["nodes"], keep, G) if gather is None else gather
    lens = torch.from_numpy(case.step["len"]).cuda()
    want = [_kv.f8(t) for t in tensors[:2]], [_kv.f64(t) for t in tensors[2:4]]
    new = kv.compact(cache, lens, torch.from_numpy(gather).cuda(), torch.tensor(keep, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert kv.device_status() == 0
    for side in range(2):
        for layer in range(case.layers):
            _kv.compact(want[0][side][layer], want[1][side][layer], case.table, case.step["len"], gather, keep, case.page)
        assert np.array_equal(_kv.f64(tensors[2 + side]), want[1][side])
        assert np.array_equal(_kv.f8(tensors[side]), want[0][side])
    assert np.array_equal(new.cpu().numpy(), case.step["len"] + np.array(keep))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_paths_across_pages(D, page):
    case = _kv.Case([0, 5, page - 1, page, 3 * page - 2, 7], [60, 33, 64, 50, 64, 64], 65, hkv=3, hq=3, D=D, page=page, layers=2, seed=page + D)
    _run(case, [5, 1, 9, 0, 21, 64], 65)


def test_whole_steps_and_consecutive_entries():
    case = _kv.Case([9, 15, 16], [40, 40, 40], 41, hkv=1, hq=1, seed=1)
    _run(case, [41, 41, 41], 41, gather=np.tile(np.arange(41, dtype=np.int32), (3, 1)))                  # nothing moves
    _run(case, [40, 40, 40], 41, gather=np.tile(np.append(np.arange(1, 41), -1).astype(np.int32), (3, 1)))   # everything by one


def test_scales_far_apart():
    """Entries that become subnormal, or vanish, beside entries of a much larger scale."""
    case = _kv.Case([3, 14], [64, 64], 65, hkv=4, hq=4, D=64, layers=3, seed=2)
    _run(case, [12, 12], 20, scales=(-30, 10))


def test_indices_out_of_order_or_range_leave_the_sequence():
    case = _kv.Case([4, 9], [12, 12], 13, layers=2, seed=3)
    kv = case.handle(binding)
    slots = case.max_pages * case.page
    for bad in ([0, 5, 5], [0, 7, 3], [-1, 2, 3], [0, 3, slots]):
        tensors = case.cache()
        before = [t.clone() for t in tensors]
        gather = np.array([bad, [0, 4, 6]], np.int32)
        new = kv.compact(binding.KVCache(*tensors), torch.tensor([4, 9], dtype=torch.int32, device="cuda"), torch.from_numpy(gather).cuda(),
                         torch.tensor([3, 3], dtype=torch.int32, device="cuda"))
        assert kv.device_status() == binding.ERR_INTERNAL
        assert new.tolist() == [4, 12]
        mine = torch.from_numpy(case.table[0]).long().cuda()
        for a, b in zip(tensors[:2], before[:2]):
            assert torch.equal(a.view(torch.uint8)[:, mine], b.view(torch.uint8)[:, mine]) and not torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for keep in (-1, 4):
        new = kv.compact(binding.KVCache(*case.cache()), torch.tensor([4, 9], dtype=torch.int32, device="cuda"),
                         torch.tensor([[0, 1, 2], [0, 1, 2]], dtype=torch.int32, device="cuda"), torch.tensor([keep, 1], dtype=torch.int32, device="cuda"))
        assert kv.device_status() == binding.ERR_INTERNAL and new.tolist() == [4, 10]


def test_new_lengths_that_overlap_what_is_read_are_refused():
    """All layers read the lengths, counts and indices while the first one writes the new lengths."""
    case = _kv.Case([4, 9, 7], [12, 12, 12], 13, layers=3, seed=4)
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    ints = torch.tensor([0, 0, 0, 4, 9, 7, 2, 3, 1, 0, 3, 5, 0, 4, 6, 0, 2, 7, 0, 0, 0], dtype=torch.int32, device="cuda")
    lens, keep, gather = ints[3:6], ints[6:9], ints[9:18].view(3, 3)
    before = ints.clone()
    for at in (1, 2, 3, 4, 6, 8, 9, 12, 17):
        with pytest.raises(binding.OptTreeError):
            kv.compact(cache, lens, gather, keep, new_len=ints[at:at + 3])
    assert kv.launch_count() == 0 and torch.equal(ints, before)
    for at in (0, 18):                                         # next to them is fine
        assert kv.compact(cache, lens, gather, keep, new_len=ints[at:at + 3]).tolist() == [6, 12, 8]
    assert kv.device_status() == 0
