"""-m gpu: the cache operators as a decoding loop uses them: with the trees, masks and keep lists that the library itself makes, in
graphs, on several streams, and over caches and batches of every size."""
import ctypes as C
import math
import struct

import numpy as np
import pytest
import torch

from paper_2406_17276_b200 import binding, synth
from tests import _kv
from tests._gpu import dev_table
from tests.test_gpu_kv_attend import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,hq,hkv,D,page", [(12, 4, 2, 64, 16), (64, 8, 2, 128, 32)])
def test_decoding_steps_with_the_librarys_own_trees(n, hq, hkv, D, page):
    """build -> mask -> (per layer: append -> attend) -> verify -> post_verify -> compact, a prompt first, several steps."""
    B, layers, V, H, depth, prompt = 3, 2, 2048, 64, 6, 37
    w = synth.Workload("kv", B, V, n, 8, depth, 3.0, 1.1, 0.3, H=H, seed=n)
    ld, lt = synth.make_tables(w)
    d_ld, d_lt = dev_table(ld), dev_table(lt)
    ot = binding.OptTree(V, H, n, w.k, depth, B)
    case = _kv.Case([0] * B, [200] * B, n + 1, hq=hq, hkv=hkv, D=D, page=page, layers=layers, tree=False, seed=n)
    kv = binding.TreeKV(hq, hkv, D, page, case.num_pages, case.max_pages, B, max(n + 1, prompt), layers=layers, dtype=case.dtype)
    cache = kv.alloc_cache(torch.from_numpy(case.table).cuda())
    angle = np.arange(400)[:, None] * 10000.0 ** (-np.arange(0, D, 2) / D)
    cs = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()
    state = lambda layer: ([_kv.f8(t)[layer] for t in (cache.k, cache.v)], [_kv.f64(t)[layer] for t in (cache.k_scale, cache.v_scale)])  # noqa: E731

    def layer_pass(layer, step, host, T):
        case.T = T
        q, k, v = case.rows(hq, 2.0), case.rows(hkv), case.rows(hkv)
        codes, scales = state(layer)
        turned = kv.append(cache, layer, q, k, v, step, cos_sin=cs)
        now, nows = state(layer)
        _kv.append(codes[1], scales[1], case.table, host, _kv.f64(v), page)         # values: exact
        assert np.array_equal(nows[1], scales[1]) and np.array_equal(now[1], codes[1])
        out = torch.full((B, T, hq, D), 77.0, dtype=case.dtype, device="cuda")
        kv.attend(cache, layer, turned, step, out=out)
        case.step = host
        check(case, out, None, (cache.k, cache.v, cache.k_scale, cache.v_scale), turned, D ** -0.5, layer)

    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    given = torch.tensor([prompt - 1, 0, prompt - 9], dtype=torch.int32, device="cuda")         # prompts of several lengths, one of a single token
    for layer in range(layers):
        layer_pass(layer, binding.KVStep(lens, given), dict(len=np.zeros(B, np.int32), nodes=given.cpu().numpy(), base=None, pos=None, mask=None), prompt)
    lens = given + 1
    roots = torch.from_numpy(synth.root_tokens(B, V, 5)).cuda()
    moved = 0
    for _ in range(4):
        tree = ot.build(d_ld, roots, -math.inf)
        mask, pos = ot.mask(tree, lens)
        step = binding.KVStep(lens, tree.n_sel, lens, pos, mask)
        host = dict(len=lens.cpu().numpy(), nodes=tree.n_sel.cpu().numpy(), base=lens.cpu().numpy(), pos=pos.cpu().numpy(), mask=mask.cpu().numpy())
        for layer in range(layers):
            layer_pass(layer, step, host, n + 1)
        alen, _, anode, roots = ot.verify(tree, d_lt, roots)
        _, gather, keep = ot.post_verify(tree, mask, alen, anode)
        want = [state(layer) for layer in range(layers)]
        new = kv.compact(cache, lens, gather, keep)
        for layer in range(layers):
            for side in range(2):
                _kv.compact(want[layer][0][side], want[layer][1][side], case.table, host["len"], gather.cpu().numpy(), keep.cpu().numpy(), page)
                assert np.array_equal(state(layer)[0][side], want[layer][0][side]) and np.array_equal(state(layer)[1][side], want[layer][1][side])
        assert torch.equal(new, lens + keep)
        moved += int((keep > 1).sum())
        lens = new
    assert moved and kv.device_status() == 0 and ot.device_status() == 0


def _problem(B, T, tree, seed, **more):
    rs = np.random.RandomState(seed)
    case = _kv.Case([int(x) for x in rs.randint(0, 300, B)], [int(x) for x in rs.randint(0, T, B)], T, tree=tree, seed=seed, **more)
    return case, case.cache(), (case.rows(case.hq), case.rows(case.hkv), case.rows(case.hkv))


@pytest.mark.parametrize("T", [1, 21, 90])
def test_captured_and_replayed(T):
    """append and attend in one graph, replayed with other lengths and rows in the same buffers; compact in another."""
    case, tensors, rows = _problem(4, T, True, T, hq=8, hkv=2, D=64)
    kv, cache, step, cs = case.handle(binding), binding.KVCache(*tensors), case.dev_step(binding), case.cos_sin(64)
    q_out, out = torch.zeros_like(rows[0]), torch.zeros_like(rows[0])
    start = [t.clone() for t in tensors]

    def call():
        kv.append(cache, 0, *rows, step, cos_sin=cs, q_out=q_out)
        kv.attend(cache, 0, q_out, step, out=out)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for change in range(3):
        if change:
            step.kv_len.copy_(torch.from_numpy(case.step["len"] // (change + 1)))
            for t in rows:
                t.copy_(case.rows(t.shape[2]))
        want = []
        for way in (call, graph.replay):
            for t, s in zip(tensors, start):
                t.view(torch.uint8).copy_(s.view(torch.uint8))
            out.zero_()
            way()
            torch.cuda.synchronize()
            want.append([t.view(torch.uint8).clone() for t in (*tensors[:4], q_out, out)])
        assert all(torch.equal(a, b) for a, b in zip(*want))
    assert kv.device_status() == 0


def test_two_handles_on_two_streams():
    """Calls that may run at the same time, each on a handle and a stream of its own, give what they give one after the other."""
    problems = []
    for seed, (T, tree) in enumerate([(1, False), (70, True), (20, True)]):
        case, tensors, rows = _problem(5, T, tree, 50 + seed, hq=8, hkv=2, D=128)
        problems.append((case, case.handle(binding), binding.KVCache(*tensors), case.dev_step(binding), rows[0]))
    alone = [kv.attend(cache, 0, q, step).clone() for _, kv, cache, step, q in problems]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    outs = [torch.zeros_like(x) for x in alone]
    torch.cuda.synchronize()
    for _ in range(20):
        for (_, kv, cache, step, q), s, o in zip(problems, streams, outs):
            with torch.cuda.stream(s):
                kv.attend(cache, 0, q, step, out=o)
    torch.cuda.synchronize()
    for (case, kv, *_), a, o in zip(problems, alone, outs):
        assert kv.device_status() == 0
        for b in range(case.B):
            m = int(case.step["nodes"][b]) + 1
            assert torch.equal(a[b, :m], o[b, :m])


def test_one_handle_for_steps_of_every_kind():
    """The same workspace serves single tokens, small and large trees in turn; repeated calls give the same bits."""
    case = _kv.Case([200, 3, 0], [89] * 3, 90, hq=8, hkv=2, D=64, seed=7)
    kv, cache = case.handle(binding), binding.KVCache(*case.cache())
    first = {}
    for turn in range(3):
        for T in (1, 2, 4, 9, 90, 1):
            g = torch.Generator(device="cuda").manual_seed(T)
            q = torch.randn((3, T, 8, 64), generator=g, device="cuda").to(case.dtype)
            out = kv.attend(cache, 0, q, binding.KVStep(torch.tensor([200, 3, 0], dtype=torch.int32, device="cuda")))
            if turn == 0:
                first.setdefault(T, out.clone())
            assert torch.equal(out, first[T])
    assert kv.device_status() == 0


@pytest.mark.parametrize("T,hq", [(1, 4), (30, 4)])
def test_more_sequences_than_are_looked_up_together(T, hq):
    case, tensors, rows = _problem(300, T, False, 60 + T, hq=hq, hkv=2, D=64, page=16)
    case.step["nodes"][::7] = -1
    kv = case.handle(binding)
    out = torch.full((300, T, hq, 64), 77.0, dtype=case.dtype, device="cuda")
    kv.attend(binding.KVCache(*tensors), 0, rows[0], case.dev_step(binding), out=out)
    assert kv.device_status() == 0
    check(case, out, None, tensors, rows[0], 64 ** -0.5)


def test_nothing_to_do():
    """A step in which no sequence takes part leaves everything as it is."""
    case, tensors, rows = _problem(3, 20, True, 8, hq=4, hkv=2, D=64)
    case.step["nodes"][:] = -1
    kv, cache, step = case.handle(binding), binding.KVCache(*tensors), case.dev_step(binding)
    before = [t.clone() for t in tensors]
    q_out, out = torch.full_like(rows[0], 77.0), torch.full_like(rows[0], 77.0)
    kv.append(cache, 0, *rows, step, cos_sin=case.cos_sin(64), q_out=q_out)
    kv.attend(cache, 0, rows[0], step, out=out)
    kv.attend(cache, 0, rows[0][:, :1].contiguous(), binding.KVStep(step.kv_len, step.nodes), out=out[:, :1].contiguous())
    assert kv.device_status() == 0
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(tensors, before))
    assert (q_out == 77.0).all() and (out == 77.0).all()


def test_offsets_beyond_32_bits():
    """Pages whose bytes lie beyond 4 GB of the cache's start."""
    page, hkv, D = 128, 8, 128
    case = _kv.Case([130, 200], [9, 4], 10, hq=16, hkv=hkv, D=D, page=page, seed=9)
    small = case.cache()
    pages = (1 << 32) // (page * hkv * D) + 40
    if torch.cuda.mem_get_info()[0] < 3 * pages * page * hkv * D:
        pytest.skip("not enough memory")
    kv = binding.TreeKV(16, hkv, D, page, pages, case.max_pages, 2, 10, dtype=case.dtype)
    k8, v8 = (torch.empty((1, pages, hkv, page, D), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.ones((1, pages, hkv), device="cuda") for _ in range(2))
    ids = torch.from_numpy(case.table).cuda().long()
    far = ids + pages - case.num_pages
    for big, t in ((k8, small[0]), (v8, small[1])):
        big.view(torch.uint8)[0, far] = t.view(torch.uint8)[0, ids]
    for big, t in ((ks, small[2]), (vs, small[3])):
        big[0, far] = t[0, ids]
    rows, step, cs = (case.rows(16), case.rows(hkv), case.rows(hkv)), case.dev_step(binding), case.cos_sin(D)
    near_kv, near = case.handle(binding), binding.KVCache(*small)
    cache = binding.KVCache(k8, v8, ks, vs, far.int())
    gather = torch.tensor([[0, 3, 8], [0, 1, 2]], dtype=torch.int32, device="cuda")
    keep = torch.tensor([3, 2], dtype=torch.int32, device="cuda")
    got = []
    for handle, c in ((near_kv, near), (kv, cache)):
        q = handle.append(c, 0, *rows, step, cos_sin=cs, q_out=torch.zeros_like(rows[0]))
        got.append((q, handle.attend(c, 0, q, step, out=torch.zeros_like(rows[0])),
                    handle.attend(c, 0, q[:, :1].contiguous(), binding.KVStep(step.kv_len), out=torch.zeros_like(rows[0][:, :1]).contiguous()),
                    handle.compact(c, step.kv_len, gather, keep)))
        assert handle.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(k8.view(torch.uint8)[0, far], small[0].view(torch.uint8)[0, ids]) and torch.equal(ks[0, far], small[2][0, ids])


def test_calls_that_are_refused():
    case, tensors, rows = _problem(2, 5, True, 10, hq=4, hkv=2, D=64)
    kv, cache, step = case.handle(binding), binding.KVCache(*tensors), case.dev_step(binding)
    q, k, v = rows
    launched = kv.launch_count()
    for bad in (dict(q=q.float()), dict(q=q[:, :, :2]), dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), dict(layer=1), dict(layer=-1),
                dict(step=binding.KVStep(step.kv_len.long())), dict(step=binding.KVStep(step.kv_len, mask=step.mask[:, :3])), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=math.nan), dict(out=torch.empty_like(q)[:, :4]), dict(lse=torch.empty((2, 5, 4), dtype=torch.float64, device="cuda")), dict(q=q.cpu()),
                dict(cache=binding.KVCache(*tensors[:4], tensors[4][:, :1].contiguous()))):
        args = dict(cache=cache, layer=0, q=q, step=step) | bad
        with pytest.raises((ValueError, binding.OptTreeError)):
            kv.attend(**args)
    cs = case.cos_sin(64)
    for bad in (dict(cos_sin=cs[:, :24].contiguous()), dict(cos_sin=torch.cat([cs, cs], 1)), dict(cos_sin=cs.double()), dict(k_norm=torch.ones(64, device="cuda")),
                dict(k_norm=torch.ones(64, dtype=case.dtype, device="cuda"), eps=math.nan), dict(k=k[:, :, :1]), dict(v=v.half()), dict(q_out=q[:, :3])):
        args = dict(cache=cache, layer=0, q=q, k=k, v=v, step=step, cos_sin=cs) | bad
        with pytest.raises((ValueError, binding.OptTreeError)):
            kv.append(**args)
    gather, keep = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (dict(kv_keep=keep[:1]), dict(kv_gather=gather.long()), dict(new_len=step.kv_len), dict(kv_gather=torch.zeros((2, 1025), dtype=torch.int32, device="cuda"))):
        with pytest.raises((ValueError, binding.OptTreeError)):
            kv.compact(**(dict(cache=cache, kv_len=step.kv_len, kv_gather=gather, kv_keep=keep) | bad))
    assert kv.launch_count() == launched and kv.device_status() == 0


def test_calls_too_large_to_count_are_refused():
    """A batch, a table and a step that together pass 2^31 tiles: refused by the sizes alone, before anything is launched."""
    cfg = binding.KVConfig(64, 64, 64, 128, 16, 1 << 23, 4096, 1, 1, 0)
    L, kv = binding.lib(), C.c_void_p()
    assert L.opt_tree_kv_create(C.byref(kv), C.byref(cfg)) == binding.OK
    some = torch.zeros(64, device="cuda").data_ptr()
    cache, rows, step = struct.pack("@5P", *[some] * 5), struct.pack("@P3q", some, 0, 0, 0), struct.pack("@2i5P", 4096, 1, some, 0, 0, 0, 0)
    assert L.opt_tree_kv_attend(kv, cache, 0, rows, step, 1.0, rows, None, None) == binding.ERR_UNSUPPORTED
    assert L.opt_tree_kv_launch_count(kv) == 0 and L.opt_tree_kv_destroy(kv) == binding.OK


def test_pointers_off_their_elements_boundary_are_refused():
    """Scales, tables, lengths, masks and sums that do not lie on a boundary of their elements would fault in a kernel."""
    case, tensors, rows = _problem(2, 5, True, 14, hq=4, hkv=2, D=64)
    kv, t = case.handle(binding), tensors
    step = case.dev_step(binding)
    L, h = binding.lib(), kv._kv
    p = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
    good_cache, good_step = [p(x) for x in t], [p(x) for x in (step.kv_len, step.nodes, step.base_pos, step.position_ids, step.mask)]
    packed = [struct.pack("@P3q", p(x), *x.stride()[:3]) for x in rows]
    lse, keep, gather, new = (torch.zeros(64, dtype=torch.float32, device="cuda") for _ in range(4))

    def attend(cache, st, sums):
        return L.opt_tree_kv_attend(h, struct.pack("@5P", *cache), 0, packed[0], struct.pack("@2i5P", 2, 5, *st), 1.0, packed[0], sums, None)

    def append(cache, st):
        return L.opt_tree_kv_append(h, struct.pack("@5P", *cache), 0, None, packed[1], packed[2], None, struct.pack("@2i5P", 2, 5, *st), None, None)

    def compact(cache, *ints):
        return L.opt_tree_kv_compact(h, struct.pack("@5P", *cache), *ints[:3], 3, 2, ints[3], None)
    ints = [p(step.kv_len), p(gather), p(keep), p(new)]
    for i in range(5):
        for by in (1, 2):
            bad = [x + by * (k == i) for k, x in enumerate(good_cache)]
            assert attend(bad, good_step, None) == append(bad, good_step) == compact(bad, *ints) == binding.ERR_INVALID_ARG
            bad = [x + (4 if i == 4 else by) * (k == i) for k, x in enumerate(good_step)]
            assert attend(good_cache, bad, None) == append(good_cache, bad) == binding.ERR_INVALID_ARG
    assert attend(good_cache, good_step, p(lse) + 2) == binding.ERR_INVALID_ARG
    for i in range(4):
        assert compact(good_cache, *[x + 2 * (k == i) for k, x in enumerate(ints)]) == binding.ERR_INVALID_ARG
    assert kv.launch_count() == 0 and kv.device_status() == 0


def test_inputs_that_ask_for_gradients_are_refused():
    """There is no backward pass: outputs would come without the gradients that were asked for."""
    case, tensors, rows = _problem(2, 5, True, 15, hq=4, hkv=2, D=64)
    kv, cache, step, cs = case.handle(binding), binding.KVCache(*tensors), case.dev_step(binding), case.cos_sin(64)
    w = torch.ones(64, dtype=case.dtype, device="cuda")
    asked = lambda t: t.clone().requires_grad_()  # noqa: E731
    q, k, v = rows
    calls = [lambda: kv.attend(cache, 0, asked(q), step), lambda: kv.attend(cache, 0, q, step, out=asked(q) * 1)]
    for i in range(3):
        calls.append(lambda i=i: kv.append(cache, 0, *[asked(t) if j == i else t for j, t in enumerate(rows)], step, cos_sin=cs))
    for name in ("q_norm", "k_norm"):
        calls.append(lambda name=name: kv.append(cache, 0, q, k, v, step, cos_sin=cs, **{name: asked(w)}))
    calls.append(lambda: kv.append(cache, 0, q, k, v, step, cos_sin=asked(cs)))
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert kv.launch_count() == 0
    with torch.no_grad():                                      # parameters of a model that serves
        for call in calls:
            call()
    assert kv.launch_count() >= len(calls) and kv.device_status() == 0
