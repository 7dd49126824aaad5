"""-m gpu: opt_tree_kv_attend against a plain 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2406_17276_b200 import binding
from tests import _kv

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def check(case, got, lse, tensors, q, scale, layer=0):
    """Tolerance: the output's rounding (half a step) and (2^-11 + 2^-12) of sum p |v|.  Probabilities may be held in half precision, whose
    11 significant bits round by up to 2^-11 of each, so that alone the sum may be off by 2^-11 of sum p |v|; single precision's errors in
    scores and sums are far below the other 2^-12 at the sizes here."""
    k, v = (_kv.f8(t)[layer] for t in tensors[:2])
    ks, vs = (_kv.f64(t)[layer] for t in tensors[2:4])
    found = _kv.attend(k, v, ks, vs, case.table, case.step, _kv.f64(q), scale, case.page)
    g, le = _kv.f64(got), None if lse is None else _kv.f64(lse)
    for b, f in enumerate(found):
        m = 0 if f is None else len(f[0])
        if f is not None:
            out, want_lse, mass = f
            tol = np.abs(out) * torch.finfo(case.dtype).eps / 2 + 2.0 ** -25 + mass * (2.0 ** -11 + 2.0 ** -12)
            bad = ~((np.abs(g[b, :m] - out) <= tol) | (np.isnan(out) & np.isnan(g[b, :m])))
            assert not bad.any(), (b, np.argwhere(bad)[:5].tolist(), float(np.nanmax(np.abs(g[b, :m] - out) / tol)))
            if le is not None:
                # scores in single precision: 2^-20 of the largest score's terms, and of the sum
                assert (np.abs(le[b, :m] - want_lse) <= 2.0 ** -18 * (1 + np.abs(want_lse)) + 2e-5).all()
        assert (g[b, m:] == 77.0).all()                                    # padding is left as it was
        if le is not None:
            assert (le[b, m:] == 77.0).all()


def run(case, pad=0, spread=2.0, scale=None, tensors=None, q=None, with_lse=True):
    kv = case.handle(binding)
    tensors = tensors or case.cache()
    q = case.rows(case.hq, spread, pad) if q is None else q
    layer = case.layers - 1
    out = torch.full((case.B, case.T, case.hq, case.D), 77.0, dtype=case.dtype, device="cuda")
    if pad:
        out = torch.full((case.B, case.T + 1, case.hq, case.D + 8 + pad), 77.0, dtype=case.dtype, device="cuda")[:, 1:, :, pad:pad + case.D]
    lse = torch.full((case.B, case.T, case.hq), 77.0, dtype=torch.float32, device="cuda") if with_lse else None
    kv.attend(binding.KVCache(*tensors), layer, q, case.dev_step(binding), scale, out, lse)
    torch.cuda.synchronize()
    assert kv.device_status() == 0 and kv.launch_count() >= 1
    check(case, out, lse, tensors, q, case.D ** -0.5 if scale is None else scale, layer)
    return out, tensors, q


@pytest.mark.parametrize("D,page,dtype", [(64, 16, BF), (64, 32, HF), (64, 64, BF), (64, 128, HF), (128, 16, HF), (128, 32, BF), (128, 64, HF), (128, 128, BF)])
def test_single_tokens(D, page, dtype):
    """Decoding: one token each, from an empty cache to a few pages, with idle sequences between."""
    run(_kv.Case([0, 1, page - 1, page, page + 1, 300, 77], [0, 0, 0, 0, 0, 0, -1], 1, D=D, page=page, dtype=dtype, hq=8, hkv=2, seed=page + D))


@pytest.mark.parametrize("D,page,dtype", [(64, 16, HF), (64, 128, BF), (128, 16, BF), (128, 32, HF), (128, 64, BF), (128, 128, HF)])
@pytest.mark.parametrize("n", [3, 10, 65, 130])
def test_trees(D, page, dtype, n):
    run(_kv.Case([0, 1, 127, 128, 200, 31], [n, n - 1, n // 2, n, 0, -1], n + 1, D=D, page=page, dtype=dtype, hq=8, hkv=2, seed=page + D + n))


@pytest.mark.parametrize("n,D,page,dtype,hq,hkv", [(300, 128, 32, BF, 6, 2), (640, 64, 16, HF, 2, 2), (1024, 128, 128, HF, 2, 1), (1024, 64, 64, BF, 3, 3)])
def test_trees_of_many_words(n, D, page, dtype, hq, hkv):
    run(_kv.Case([5, 0, 260, 1000], [n, n // 2 + 1, 63, 64], n + 1, D=D, page=page, dtype=dtype, hq=hq, hkv=hkv, seed=n + D))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (7, 1), (12, 4), (16, 1), (33, 1), (64, 2), (5, 5)])
def test_heads(hq, hkv):
    run(_kv.Case([100, 9], [0, 0], 1, hq=hq, hkv=hkv, D=128, seed=hq))
    run(_kv.Case([100, 9], [9, 20], 21, hq=hq, hkv=hkv, D=64, seed=hq))


@pytest.mark.parametrize("T", [2, 17, 129, 257, 300])
def test_chains(T):
    run(_kv.Case([0, 5, 140], [T - 1, T - 1, T // 2], T, tree=False, hq=4, hkv=2, D=128, page=32, seed=T))
    run(_kv.Case([0, 133], [T - 1, T - 1], T, tree=False, hq=3, hkv=3, D=64, page=16, dtype=HF, seed=T))


@pytest.mark.parametrize("length", [1000, 4097, 20000])
def test_long_prefixes(length):
    run(_kv.Case([length, length // 3], [0, 0], 1, hq=4, hkv=1, D=128, page=64, seed=length))
    run(_kv.Case([length, 17], [20, 11], 21, hq=4, hkv=2, D=64, page=16, seed=length))


def test_many_ragged_sequences():
    rs = np.random.RandomState(3)
    lens = [int(x) for x in rs.randint(0, 700, 40)]
    run(_kv.Case(lens, [int(x) for x in rs.randint(-1, 13, 40)], 13, hq=6, hkv=2, D=64, page=32, seed=4))
    run(_kv.Case(lens, [int(x) for x in rs.randint(-1, 1, 40)], 1, hq=8, hkv=4, D=128, page=16, seed=5))


@pytest.mark.parametrize("pad", [1, 4, 8])
def test_strided_rows_on_any_boundary(pad):
    run(_kv.Case([30, 7], [4, 6], 7, seed=pad), pad=pad)
    run(_kv.Case([30, 7], [0, 0], 1, D=128, dtype=HF, seed=pad), pad=pad)
    run(_kv.Case([30, 7], [140, 90], 141, D=128, dtype=HF, seed=pad), pad=pad)


def test_without_lse_other_scale_and_last_layer():
    run(_kv.Case([30, 7], [4, 6], 7, layers=3, seed=1), with_lse=False, scale=0.03)


@pytest.mark.parametrize("T,hq,hkv", [(1, 4, 2), (9, 4, 2), (70, 8, 2), (150, 4, 1)])
def test_unwritten_slots_and_pages(T, hq, hkv):
    """Whatever lies behind a sequence's last slot, and in pages of no sequence, NaN codes and NaN scales included, stays out; table
    entries behind the last page are not looked at."""
    case = _kv.Case([20, 3, 128], [T - 1, T // 2, T - 1], T, hq=hq, hkv=hkv, D=64, seed=T)
    tensors = case.cache()
    used = torch.zeros((case.num_pages, case.page), dtype=torch.bool, device="cuda")
    table = case.table.copy()
    for b in range(3):
        end = int(case.step["len"][b] + case.step["nodes"][b]) + 1
        for s in range(end):
            used[int(case.table[b, s // case.page]), s % case.page] = True
        table[b, (end - 1) // case.page + 1:] = 1 << 30
    for t in tensors[:2]:
        t.view(torch.uint8)[0].masked_fill_(~used[:, None, :, None], 0x7F)
    for t in tensors[2:4]:
        t[0].masked_fill_(~used.any(1)[:, None], float("nan"))
    tensors[4].copy_(torch.from_numpy(table))
    run(case, tensors=tensors)


@pytest.mark.parametrize("T,hq,hkv", [(9, 4, 2), (70, 8, 2), (150, 4, 1)])
def test_nan_of_one_node_reaches_only_those_who_see_it(T, hq, hkv):
    case = _kv.Case([20, 0], [T - 1, T - 1], T, hq=hq, hkv=hkv, D=64, seed=T)
    tensors = case.cache()
    for side, j in ((0, T - 1), (1, 2), (1, T // 2)):
        for b in range(2):
            s = int(case.step["len"][b]) + j
            tensors[side].view(torch.uint8)[0, int(case.table[b, s // case.page]), :, s % case.page, 5] = 0x7F
    out, *_ = run(case, tensors=tensors, with_lse=False)
    assert torch.isnan(out.float()).any() and torch.isfinite(out.float()).any()


def test_scores_of_every_size():
    """Queries so large that one key takes all, and so small that all keys weigh the same; zero queries."""
    for spread in (1000.0, 1e-4, 0.0):
        run(_kv.Case([150, 40], [6, 6], 7, D=128, dtype=BF, seed=7), spread=spread)
        run(_kv.Case([150, 40], [0, 0], 1, D=64, dtype=HF, seed=8), spread=spread)
        run(_kv.Case([150, 40], [60, 40], 61, D=128, hq=8, hkv=2, seed=9), spread=spread)


def test_queries_of_the_whole_range_of_the_type():
    """bf16 rows of 1e30 and of 1e-30 in one call."""
    case = _kv.Case([70, 9], [5, 5], 6, D=64, seed=10)
    q = case.rows(case.hq)
    q[0] *= 1e30
    q[1] *= 1e-30
    tensors = case.cache()
    tensors[2].fill_(2.0 ** -20)
    run(case, q=q, tensors=tensors, scale=1e-24)


@pytest.mark.parametrize("T", [1, 7, 80])
def test_scales_far_apart(T):
    """Pages whose scales differ by 2^12: small pages keep their part of the sum."""
    case = _kv.Case([170, 60], [T - 1, T // 2], T, D=64, hq=8, hkv=2, seed=11)
    run(case, tensors=case.cache(scales=(-14, -2)), spread=0.05)


def test_scales_that_are_no_powers_of_two():
    case = _kv.Case([90, 60], [6, 2], 7, D=64, hq=8, hkv=2, seed=12)
    tensors = case.cache()
    for t in tensors[2:4]:
        t.mul_(1.37)
    run(case, tensors=tensors)


def test_shared_prefix_pages():
    """Two sequences whose tables name the same pages for the prefix."""
    case = _kv.Case([64, 64, 64], [6, 3, 0], 7, page=16, seed=13)
    case.table[1:, :4] = case.table[0, :4]
    run(case)


def test_sizes_and_pages_out_of_range_are_recorded():
    case = _kv.Case([40, 9], [3, 3], 4, seed=14)
    kv, q = case.handle(binding), case.rows(4)
    for change in ("page", "len", "nodes", "negative"):
        tensors, step = case.cache(), case.dev_step(binding)
        if change == "page":
            tensors[4][0, 1] = -5
        elif change == "len":
            step.kv_len[0] = case.max_pages * case.page
        elif change == "nodes":
            step.nodes[0] = case.T
        else:
            step.kv_len[0] = -1
        out = torch.full((2, 4, 4, 64), 77.0, dtype=case.dtype, device="cuda")
        kv.attend(binding.KVCache(*tensors), 0, q, step, None, out)
        assert kv.device_status() == binding.ERR_INTERNAL and kv.device_status() == 0
        assert torch.isfinite(out[1].float()).all() and not (out[1] == 77.0).any()          # the other sequence is served


@pytest.mark.parametrize("tiles", [2, 3, 4, 5, 7])
@pytest.mark.parametrize("B,hkv", [(1, 1), (60, 4)])
def test_nan_values_in_every_key_tile_of_a_single_row_tile(tiles, B, hkv):
    """70 rows per key head, a step that lies in the last two tiles of 128 keys: whichever of the two groups takes the NaN, and whether
    the row tile is cut or not, the rows that see it are NaN and no others."""
    T = 70
    case = _kv.Case([128 * (tiles - 1) - 30 + b % 2 * 35 for b in range(B)], [T - 1] * B, T, hq=hkv, hkv=hkv, D=64, page=32, seed=tiles)
    tensors = case.cache()
    for j in (3, 68):                                          # the first one before the last tile, in every other sequence
        for b in range(B):
            s = int(case.step["len"][b]) + j
            tensors[1].view(torch.uint8)[0, int(case.table[b, s // case.page]), :, s % case.page, 5 + j % 2] = 0x7F
    q = case.rows(case.hq, 2.0)
    for _ in range(5):
        run(case, tensors=tensors, q=q, with_lse=False)


@pytest.mark.parametrize("T", [1, 7, 30, 80, 150])
@pytest.mark.parametrize("side,spread", [("both", 2.0), ("keys", 4.0), ("values", 1.0)])
def test_scales_with_a_fraction_of_their_own(T, side, spread):
    """Every page and head has a scale of its own that is no power of two: both kernels, single and double row tiles."""
    for D, hq, hkv in ((64, 8, 2), (128, 3, 3)):
        case = _kv.Case([290, 60, 7], [T - 1, T // 2, T - 1], T, D=D, hq=hq, hkv=hkv, seed=20 + T)
        tensors = case.cache()
        for which, t in (("keys", tensors[2]), ("values", tensors[3])):
            if side in ("both", which):
                t.mul_(torch.from_numpy(case.rs.uniform(1.0, 2.0, tuple(t.shape))).float().cuda())
        run(case, tensors=tensors, spread=spread)


def test_largest_and_smallest_scales():
    """Scales above 2^127 and below 2^-126 (values 0 and tiny codes where the scale is huge, so that outputs are finite)."""
    for T in (1, 90):
        case = _kv.Case([150, 40], [T - 1, T // 3], T, D=64, hq=4, hkv=2, seed=30 + T)
        tensors = case.cache(spread=2.0 ** -7)
        tensors[2].fill_(2.0 ** -127)
        tensors[3].fill_(1.5 * 2.0 ** 127)
        run(case, tensors=tensors)
