"""-m gpu: opt_tree_kv_append against a plain 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2406_17276_b200 import binding
from tests import _kv

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def _run(case, rot=None, interleaved=False, norm=False, pad=0, eps=1e-5, with_q=True, rows=None, older=True):
    kv = case.handle(binding)
    k8, v8, ks, vs, table = case.cache()
    cache = binding.KVCache(k8, v8, ks, vs, table)
    layer = case.layers - 1
    D = case.D
    rot = D if rot is None else rot
    q, k, v = rows if rows else (case.rows(case.hq, 2.0, pad), case.rows(case.hkv, 1.5, pad), case.rows(case.hkv, 0.7, pad))
    w = [(1 + 0.3 * torch.from_numpy(case.rs.standard_normal(D))).to(case.dtype).cuda() for _ in range(2)] if norm else [None, None]
    cs = case.cos_sin(rot) if rot else None
    before = [_kv.f8(t) for t in (k8, v8)], [_kv.f64(t) for t in (ks, vs)]
    q_out = torch.full((case.B, case.T, case.hq, D), 77.0, dtype=case.dtype, device="cuda")
    got = kv.append(cache, layer, q if with_q else None, k, v, case.dev_step(binding), cos_sin=cs, q_norm=w[0], k_norm=w[1], eps=eps,
                    interleaved=interleaved, q_out=q_out if with_q else None)
    torch.cuda.synchronize()
    assert kv.device_status() == 0 and kv.launch_count() == 1
    # the plain form
    csn = None if cs is None else _kv.f64(cs)
    pos = [_kv.positions(case.step, b, int(case.step["nodes"][b]) + 1) for b in range(case.B)]

    def turn(x, weight):
        x = _kv.f64(x)
        for b in range(case.B):
            m = len(pos[b])
            if m:
                x[b, :m] = _kv.turned(x[b, :m], None if weight is None else _kv.f64(weight), eps, None if csn is None else csn[pos[b]][:, None], rot, interleaved)
        return x
    if with_q:
        want, g = turn(q, w[0]), _kv.f64(got)
        mag = np.abs(want).max(-1, keepdims=True)
        for b in range(case.B):
            m = len(pos[b])
            # one rounding to the type (half a step), and single precision before it: a few 2^-24 of the row's largest value
            half = np.maximum(np.abs(want[b, :m]) * torch.finfo(case.dtype).eps / 2, 2.0 ** -25)
            assert (np.abs(g[b, :m] - want[b, :m]) <= half + 2e-6 * mag[b, :m]).all()
            assert (g[b, m:] == 77.0).all()                                    # padding is left as it was
    for side, (x, t, sc) in enumerate(((turn(k, w[1]), k8, ks), (_kv.f64(v), v8, vs))):
        codes, scale = before[0][side], before[1][side]
        _kv.append(codes[layer], scale[layer], case.table, case.step, x, case.page)
        now, nows = _kv.f8(t), _kv.f64(sc)
        assert np.array_equal(nows, scale)
        # the new entries (roundings of exact values) and the other rows, pages and layers
        assert np.array_equal(now, codes, equal_nan=True)
    return kv


@pytest.mark.parametrize("D,page,dtype", [(64, 16, BF), (64, 32, HF), (64, 64, BF), (64, 128, HF), (128, 16, HF), (128, 32, BF), (128, 64, HF), (128, 128, BF)])
@pytest.mark.parametrize("norm,interleaved", [(False, False), (True, True), (True, False)])
def test_pages_and_styles(D, page, dtype, norm, interleaved):
    _run(_kv.Case([0, 1, page - 1, page, 3 * page + 5, 37], [0, 4, 11, 2, 11, -1], 12, D=D, page=page, dtype=dtype, seed=page + D), norm=norm, interleaved=interleaved)


@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (32, False), (96, False), (112, False), (16, True), (96, True)])
def test_partly_rotated_rows(rot, interleaved):
    _run(_kv.Case([5, 40], [6, 3], 7, D=128, seed=rot), rot=rot, interleaved=interleaved, norm=True)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 1), (6, 3), (32, 8), (5, 5)])
def test_heads(hq, hkv):
    _run(_kv.Case([9, 0, 31], [20, 3, 17], 21, hq=hq, hkv=hkv, D=128, seed=hq), norm=True)


@pytest.mark.parametrize("pad", [1, 4, 8])
def test_strided_rows_on_any_boundary(pad):
    _run(_kv.Case([3, 17], [4, 6], 7, D=64, seed=pad), norm=True, pad=pad)
    _run(_kv.Case([3, 17], [4, 6], 7, D=128, dtype=HF, seed=pad), interleaved=True, pad=pad)


def test_chain_across_pages_and_single_tokens():
    _run(_kv.Case([0, 13], [200, 150], 201, tree=False, page=16, seed=1))
    _run(_kv.Case([0, 13], [200, 150], 201, tree=False, page=128, D=128, seed=2), norm=True)
    _run(_kv.Case([0, 15, 16, 63], [0, 0, 0, -1], 1, page=16, seed=3))


def test_without_queries_and_in_the_last_of_several_layers():
    _run(_kv.Case([0, 13], [4, 2], 5, seed=4, layers=3), with_q=False)


def test_queries_in_place():
    case = _kv.Case([4, 9], [4, 1], 5, seed=5)
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    q, k, v = case.rows(case.hq), case.rows(case.hkv), case.rows(case.hkv)
    cs, step = case.cos_sin(64), case.dev_step(binding)
    apart = kv.append(cache, 0, q, k, v, step, cos_sin=cs, q_out=q.clone())
    kv.append(cache, 0, q, k, v, step, cos_sin=cs, q_out=q)
    assert torch.equal(apart, q)


def test_values_on_the_borders_of_scales_and_codes():
    """Largest values of 448 * 2^j exactly and one step above, ties between codes, zeros, and values below the smallest scale."""
    case = _kv.Case([0, 16, 5, 0, 0], [3, 3, 3, 3, 3], 4, hq=2, hkv=2, D=64, seed=6)
    k, v = case.rows(2), case.rows(2)
    for t in (k, v):
        t[0, 0, 0, 0], t[0, 0, 1, 0] = 448.0, 450.0
        t[1, 0, 0, 5], t[1, 0, 1, 5] = 1.75, -1.7578125
        t[2] = 0
        t[3] = torch.linspace(16.0, 18.0, 64, device="cuda").to(case.dtype)      # steps of a quarter code: ties among them
        t[4] = 2.0 ** -80
    _run(case, rot=0, rows=(case.rows(2), k, v))
    _run(case, rot=64, norm=True, rows=(case.rows(2), k, v))


def test_borders_that_single_precision_cannot_see():
    """Normed keys whose largest value is 448 * 2^j up to the last bits of a double: the scale is that of exact arithmetic."""
    case = _kv.Case([0] * 8, [1] * 8, 2, hq=2, hkv=2, D=64, tree=False, seed=7)
    k = case.rows(2)
    k[:] = 1.0                                # norm of ones is 1 / sqrt(1 + eps), the weight below brings the largest to 1.75 * that
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    w = torch.full((64,), 1.75, dtype=case.dtype, device="cuda")
    for eps, want in ((0.0, 2.0 ** -8), (1e-12, 2.0 ** -8), (-1.0, None)):
        if eps < 0:
            with pytest.raises(binding.OptTreeError):
                kv.append(cache, 0, None, k, k, case.dev_step(binding), k_norm=w, eps=eps)
            continue
        kv.append(cache, 0, None, k, k, case.dev_step(binding), k_norm=w, eps=eps)
        ids = case.table[:, 0]
        assert (_kv.f64(cache.k_scale)[0, ids] == want).all()


def test_infinities_and_nan():
    """Infinities saturate, NaN stays NaN, and neither sets the scale."""
    case = _kv.Case([3, 0], [3, 3], 4, hq=2, hkv=2, D=64, seed=8)
    k, v = case.rows(2), case.rows(2)
    for t in (k, v):
        t[0, 1, 0, 3], t[0, 2, 1, 7], t[0, 2, 1, 8] = float("inf"), float("-inf"), float("nan")
        t[1] = float("nan")
    _run(case, rot=0, rows=(case.rows(2), k, v))


def test_older_entries_keep_their_values_when_the_scale_grows():
    """A page filled token by token with growing values: what was stored is brought along exactly (powers of two)."""
    case = _kv.Case([0], [0], 1, hq=1, hkv=1, D=64, page=16, seed=9)
    kv = case.handle(binding)
    cache = binding.KVCache(*case.cache())
    rows = []
    for t in range(12):
        x = (case.rows(1) * 1.5 ** t).to(case.dtype)
        step = binding.KVStep(torch.tensor([t], dtype=torch.int32, device="cuda"))
        kv.append(cache, 0, None, x, x, step)
        s = float(cache.k_scale[0, case.table[0, 0], 0])
        old = np.array(rows[:])
        now = _kv.f8(cache.k)[0, case.table[0, 0], 0, :t + 1] * s
        if t:
            fine = np.abs(old) >= 2.0 ** -6 * s                                # still normal numbers
            assert np.array_equal(now[:t][fine], old[fine])
            assert (np.abs(now[:t] - old) <= 2.0 ** -10 * s).all()             # else half a subnormal step
        rows = list(now)


def test_positions_and_pages_out_of_range_are_recorded():
    case = _kv.Case([4, 9], [3, 3], 4, seed=10)
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    rows = (case.rows(4), case.rows(2), case.rows(2))
    kv.append(cache, 0, *rows, case.dev_step(binding), cos_sin=case.cos_sin(64)[:6])
    assert kv.device_status() == binding.ERR_INTERNAL and kv.device_status() == 0
    # a page that does not exist, lengths that do not fit: the sequence is left out, the other one is served
    for change in ("page", "len", "nodes", "negative"):
        k8, v8, ks, vs, table = case.cache()
        cache, step = binding.KVCache(k8, v8, ks, vs, table), case.dev_step(binding)
        if change == "page":
            table[0, 0] = case.num_pages
        elif change == "len":
            step.kv_len[0] = case.max_pages * case.page - 3
        elif change == "nodes":
            step.nodes[0] = case.T
        else:
            step.kv_len[0] = -1
        before = k8.view(torch.uint8).clone()
        kv.append(cache, 0, *rows, step, cos_sin=case.cos_sin(64))
        assert kv.device_status() == binding.ERR_INTERNAL
        now = k8.view(torch.uint8)
        other = torch.tensor(case.table[1], device="cuda").long()
        rest = torch.ones(case.num_pages, dtype=torch.bool, device="cuda")
        rest[other] = False
        assert torch.equal(now[0, rest], before[0, rest]) and not torch.equal(now, before)


@pytest.mark.parametrize("D,page,rot,interleaved", [(64, 16, 64, False), (128, 32, 128, True), (128, 128, 0, False), (64, 64, 32, False)])
def test_norms_of_the_whole_range_of_the_type(D, page, rot, interleaved):
    """bf16 rows whose squares pass single precision's range at either end, beside ordinary ones: queries, scales and codes."""
    for eps in (0.0, 1e-5):
        case = _kv.Case([5, 0, page, 3], [6, 6, 6, 6], 7, hq=4, hkv=2, D=D, page=page, seed=D + page)
        q, k, v = case.rows(4), case.rows(2), case.rows(2)
        for t in (q, k):
            t[0] *= 1e25
            t[1] *= 1e-25
            t[2, ::2] *= 1e-30
            t[2, 1::2] *= 1e19
            t[3, 2, 1, 3] = 3e38
            t[3, 4, 0] = 3e38
            t[3, 5, 1] *= 1e-10
        _run(case, rot=rot, interleaved=interleaved, norm=True, eps=eps, rows=(q, k, v))


def test_norm_weights_of_the_whole_range_of_the_type():
    """Products that pass single precision's range on the way to an ordinary result, and keys beyond that range."""
    case = _kv.Case([5, 0], [6, 6], 7, hq=4, hkv=2, D=64, seed=11)
    q, k, v = case.rows(4, 1e15), case.rows(2, 1e15), case.rows(2)
    kv, cache, cs = case.handle(binding), binding.KVCache(*case.cache()), case.cos_sin(64)
    w = (1e30 * (1 + torch.rand(64, generator=torch.Generator().manual_seed(1)))).to(case.dtype).cuda()
    codes, scale = _kv.f8(cache.k)[0], _kv.f64(cache.k_scale)[0]
    got = kv.append(cache, 0, q, k, v, case.dev_step(binding), cos_sin=cs, q_norm=w, k_norm=w, eps=0.0)
    turn = lambda x: np.stack([_kv.turned(_kv.f64(x)[b], _kv.f64(w), 0.0, _kv.f64(cs)[_kv.positions(case.step, b, 7)][:, None], 64, False) for b in range(2)])  # noqa: E731
    want = turn(q)
    assert (np.abs(_kv.f64(got) - want) <= np.abs(want) * 2.0 ** -8 + 2e-6 * np.abs(want).max(-1, keepdims=True)).all()
    _kv.append(codes, scale, case.table, case.step, turn(k), case.page)
    assert np.array_equal(_kv.f64(cache.k_scale)[0], scale) and np.array_equal(_kv.f8(cache.k)[0], codes)
    # rotation alone, of values near the type's largest: pairs sum to more than single precision holds
    case = _kv.Case([5, 0], [6, 6], 7, hq=4, hkv=2, D=64, seed=12)
    k = (3.3e38 * torch.sign(case.rows(2).float())).to(case.dtype)
    _run(case, rot=64, rows=(case.rows(4), k, case.rows(2)), with_q=False)


@pytest.mark.parametrize("rot,interleaved", [(16, False), (48, False), (16, True), (48, True)])
@pytest.mark.parametrize("D,dtype", [(64, BF), (128, HF)])
def test_infinities_and_nan_behind_the_rotated_part(rot, interleaved, D, dtype):
    """Elements that are not rotated come through as they are, and do not reach their neighbours; rotated ones saturate."""
    case = _kv.Case([3, 0], [3, 3], 4, hq=2, hkv=2, D=D, dtype=dtype, seed=rot + D)
    q, k, v = (case.rows(2) for _ in range(3))
    for t in (q, k):
        t[0, 1, 0, rot + 3], t[0, 2, 1, rot + 7], t[0, 2, 1, D - 1] = float("inf"), float("-inf"), float("nan")
        t[0, 3, 0, rot + 2] = float("inf")
    k[0, 3, 0, 5] = float("inf")
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    got = kv.append(cache, 0, q, k, v, case.dev_step(binding), cos_sin=case.cos_sin(rot), interleaved=interleaved)
    assert np.array_equal(_kv.f64(got[..., rot:]), _kv.f64(q[..., rot:]), equal_nan=True) and torch.isfinite(got[..., :rot].float()).all()
    _run(case, rot=rot, interleaved=interleaved, rows=(q, k, v), with_q=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rot", [None, 32])
def test_queries_in_place_beside_rows_that_are_taken_again(D, rot):
    """Rows of 1e25 between ordinary ones of the same token: in place as apart."""
    case = _kv.Case([4, 9], [4, 4], 5, hq=10, hkv=2, D=D, seed=D)
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    q, k, v = case.rows(10), case.rows(2), case.rows(2)
    for h in (0, 3, 6, 9):
        q[:, h % 5, h] *= 1e25
    w = (1 + 0.3 * torch.from_numpy(case.rs.standard_normal(D))).to(case.dtype).cuda()
    more = dict(cos_sin=case.cos_sin(rot or D), q_norm=w, k_norm=w)
    apart = kv.append(cache, 0, q, k, v, case.dev_step(binding), q_out=torch.zeros_like(q), **more)
    kv.append(cache, 0, q, k, v, case.dev_step(binding), q_out=q, **more)
    assert torch.equal(apart, q) and apart.float().abs().max() < 100
