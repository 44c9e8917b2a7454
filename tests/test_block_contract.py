"""The operators around attention under the contract of the library's calls: recorded into a graph and replayed on new data, on other
streams and from two threads, poisoned margins around everything they write, tensors beyond 2^31 elements."""
import threading

import pytest
import torch

from tests import _block as B
from tests.test_guard_bands import Guarded

pytestmark = pytest.mark.gpu
T, HQ, HKV, D, C = 1501, 4, 2, 80, 1280


def _data(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    cuts = torch.randint(1, T, (5,), generator=gen, device="cuda").sort().values.int()
    edge = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    return dict(x=normal(T, C), r=normal(T, C), w=normal(C), b=normal(C), qkv=normal(T, HQ + 2 * HKV, D), dy=normal(T, C), ds=normal(T, C),
                do=normal(T, HQ, D), cu=torch.cat([edge[:1], cuts, edge[1:]]),
                grids=torch.randint(0, 9, (6, 3), generator=gen, device="cuda", dtype=torch.int32) * 2,
                first=torch.randint(0, 99, (6,), generator=gen, device="cuda", dtype=torch.int32),
                freq=torch.rand(D // 2, generator=gen, device="cuda"), axis=torch.randint(0, 3, (D // 2,), generator=gen, device="cuda", dtype=torch.int32))


def _all(binding, d, fmt="int8", **on):
    """Every entry point once, as a training step would; all results."""
    f = binding.varlen_attn_norm_fwd(d["x"], d["w"], d["b"], residual=d["r"], save=fmt, **on)
    pos = binding.varlen_attn_rotary_positions(d["cu"], d["grids"], T, first=d["first"], merge=2, **on)
    turn = (pos, d["freq"], d["axis"])
    qkv = d["qkv"]
    q, k, v = binding.varlen_attn_rotary_fwd(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], *turn, v=qkv[:, HQ + HKV:], **on)
    o, lse = binding.varlen_attn_fwd(q, k, v, d["cu"], True, 0.1, kv_splits=1, **on)
    kept = binding.varlen_attn_act8_pack([q, k, v, o], fmt, **on)
    back = binding.varlen_attn_act8_unpack(kept, **on)
    dq, dk, dv = binding.varlen_attn_bwd_act8(d["do"], *kept, lse, d["cu"], True, 0.1, kv_splits=1, **on)
    grads = torch.empty_like(qkv)
    binding.varlen_attn_rotary_bwd(dq, dk, *turn, dv=dv, dq_out=grads[:, :HQ], dk_out=grads[:, HQ:HQ + HKV], dv_out=grads[:, HQ + HKV:], **on)
    dx, dw, db = binding.varlen_attn_norm_bwd(d["dy"], f.saved, f.mean, f.rstd, d["w"], dsummed=d["ds"], **on)
    return [f.out, f.mean, f.rstd, f.summed, *f.saved, pos, q, k, v, o, lse, *(t for x in kept for t in x), *back, dq, dk, dv, grads, dx, dw, db]


def _same(a, b):
    bits = lambda t: t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t  # noqa: E731
    assert len(a) == len(b)
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(bits(x), bits(y)), i


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_recorded_once_and_replayed_on_new_data(fmt):
    from paper_2605_08962_amd import binding
    d = _data(1)
    _all(binding, d, fmt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _all(binding, d, fmt)
    for seed in (2, 3, 4, 5):
        new = _data(seed)
        for n, t in d.items():
            t.copy_(new[n])
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        _same(got, _all(binding, new, fmt))
        torch.cuda.synchronize()


def test_two_graphs_keep_out_of_each_others_way():
    """Recorded one after the other, replayed in turns on two streams: no scratch of one is the other's."""
    from paper_2605_08962_amd import binding
    sets, graphs, got = [_data(11), _data(12)], [], []
    want = [[t.clone() for t in _all(binding, d)] for d in sets]
    torch.cuda.synchronize()
    for d in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(_all(binding, d))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            _same(a, b)


def test_another_stream():
    """Named by the call, or current: the results of the current stream's calls, allocated in the stream's pool."""
    from paper_2605_08962_amd import binding
    d = _data(6)
    want = _all(binding, d)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = _all(binding, d, stream=side)
    torch.cuda.synchronize()
    _same(got, want)
    segments = [(s["address"], s["address"] + s["total_size"]) for s in torch.cuda.memory_snapshot() if s["stream"] == side.cuda_stream]
    for t in got[:1] + got[4:8]:
        assert any(a <= t.data_ptr() < b for a, b in segments)
    with torch.cuda.stream(side):
        got = _all(binding, d)
    torch.cuda.synchronize()
    _same(got, want)


def test_two_host_threads():
    from paper_2605_08962_amd import binding
    sets = [_data(21), _data(22)]
    want = [_all(binding, d) for d in sets]
    torch.cuda.synchronize()
    results = [None, None]

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                results[i] = _all(binding, sets[i])
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for a, b in zip(results, want):
        _same(a, b)


@pytest.mark.parametrize("T,C", [(301, 1280), (77, 1001), (5, 64), (130, 8200), (9, 16384)])
def test_margins_of_the_norm(T, C):
    from paper_2605_08962_amd import binding
    x, dy, w = B.bf(T, C, seed=1), B.bf(T, C, seed=2), B.bf(C, seed=3)
    f = binding.varlen_attn_norm_fwd(x, w, save="int8", residual=x)
    p = binding.NormParams(T, 1, C, 0, 0, 1e-5, C, C, C)
    g = {n: Guarded(size) for n, size in (("y", 2 * T * C), ("summed", 2 * T * C), ("mean", 4 * T), ("rstd", 4 * T), ("codes", T * C),
                                          ("scales", 4 * f.saved.scales.numel()), ("dx", 2 * T * C), ("dw", 4 * C), ("db", 4 * C),
                                          ("ws", binding.norm_bwd_workspace_bytes(p)))}
    ptr = {n: b.bytes_view().data_ptr() for n, b in g.items()}
    import ctypes
    lib, s = binding.load(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    assert lib.varlen_attn_norm_fwd(ctypes.byref(p), x.data_ptr(), x.data_ptr(), w.data_ptr(), None, ptr["y"], ptr["summed"], ptr["mean"],
                                    ptr["rstd"], ptr["codes"], ptr["scales"], s) == 0
    assert lib.varlen_attn_norm_bwd(ctypes.byref(p), dy.data_ptr(), None, ptr["codes"], ptr["scales"], ptr["mean"], ptr["rstd"], w.data_ptr(),
                                    None, ptr["dx"], ptr["dw"], ptr["db"], ptr["ws"], g["ws"].n, s) == 0
    torch.cuda.synchronize()
    for n, b in g.items():
        assert b.intact(), n
    assert torch.equal(g["y"].view(torch.bfloat16, (T, C)), f.out) and torch.equal(g["codes"].view(torch.int8, (T, C)), f.saved.codes)
    want = binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd, w)
    assert torch.equal(g["dx"].view(torch.bfloat16, (T, C)), want[0]) and torch.equal(g["dw"].view(torch.float32, (C,)), want[1])


@pytest.mark.parametrize("T,hq,hkv,d,P,interleaved", [(301, 4, 2, 64, 32, False), (5, 3, 1, 80, 40, False), (77, 2, 2, 128, 64, False),
                                                      (33, 2, 1, 96, 48, True), (9, 1, 1, 7, 3, False), (41, 2, 1, 80, 20, False)])
def test_margins_of_rotary_and_packing(T, hq, hkv, d, P, interleaved):
    from paper_2605_08962_amd import binding
    q, k = B.bf(T, hq, d, seed=1), B.bf(T, hkv, d, seed=2)
    pos = torch.randint(0, 99, (2, T), dtype=torch.int32, device="cuda")
    freq, axis = torch.rand(P, device="cuda"), torch.zeros(P, dtype=torch.int32, device="cuda")
    sizes = [2 * t.numel() for t in (q, k, k)]
    g = [Guarded(n) for n in sizes]
    outs = [b.view(torch.bfloat16, t.shape) for b, t in zip(g, (q, k, k))]
    binding.varlen_attn_rotary_fwd(q, k, pos, freq, axis, v=k, interleaved=interleaved, q_out=outs[0], k_out=outs[1], v_out=outs[2])
    want = binding.varlen_attn_rotary_fwd(q, k, pos, freq, axis, v=k, interleaved=interleaved)
    packed = binding.varlen_attn_act8_pack([q, k])
    g8 = [Guarded(t.numel() * t.element_size()) for x in packed for t in x]
    mine = [binding.Act8(g8[2 * i].view(x.codes.dtype, x.codes.shape), g8[2 * i + 1].view(torch.float32, x.scales.shape)) for i, x in enumerate(packed)]
    binding.varlen_attn_act8_pack([q, k], out=mine)
    gu = [Guarded(2 * t.numel()) for t in (q, k)]
    binding.varlen_attn_act8_unpack(packed, out=[b.view(torch.bfloat16, t.shape) for b, t in zip(gu, (q, k))])
    torch.cuda.synchronize()
    assert all(b.intact() for b in g + g8 + gu)
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert all(torch.equal(a, b) for x, y in zip(mine, packed) for a, b in zip(x, y))


def test_tensors_beyond_two_to_the_31_elements():
    """Rows at both ends and around element 2^31, against the same rows by themselves."""
    from paper_2605_08962_amd import binding
    T, h, d = 1_050_007, 16, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((T, h, d), dtype=torch.bfloat16, device="cuda")
    for at in range(0, T, 100_000):
        n = min(100_000, T - at)
        x[at:at + n] = torch.randn((n, h, d), generator=gen, device="cuda").to(torch.bfloat16)
    assert x.numel() > 2 ** 31
    mid = 2 ** 31 // (h * d)
    rows = [slice(0, 64), slice(mid - 32, mid + 32), slice(T - 64, T)]
    pos = torch.arange(T, dtype=torch.int32, device="cuda").expand(2, -1).contiguous()
    freq, axis = torch.rand(64, device="cuda"), (torch.arange(64, device="cuda") % 2).int()
    print("rotary", flush=True)
    y = binding.varlen_attn_rotary_fwd(x[:, :12], x[:, 12:14], pos, freq, axis, v=x[:, 14:])
    for s in rows:
        want = binding.varlen_attn_rotary_fwd(x[s, :12], x[s, 12:14], pos[:, s].contiguous(), freq, axis, v=x[s, 14:])
        assert all(torch.equal(a[s], b) for a, b in zip(y, want))
    del y
    print("act8", flush=True)
    packed = binding.varlen_attn_act8_pack([x])[0]
    for s in rows:
        want = binding.varlen_attn_act8_pack([x[s]])[0]
        assert torch.equal(packed.codes[s], want.codes) and torch.equal(packed.scales[s], want.scales)
    back = binding.varlen_attn_act8_unpack([packed])[0]
    for s in rows:
        assert torch.equal(back[s], binding.varlen_attn_act8_unpack([binding.Act8(packed.codes[s], packed.scales[s])])[0])
    del back
    print("norm", flush=True)
    w = torch.rand(h * d, device="cuda")
    flat = x.view(T, h * d)
    f = binding.varlen_attn_norm_fwd(flat, w, save="int8")
    dx, dw, db = binding.varlen_attn_norm_bwd(flat, f.saved, f.mean, f.rstd, w)
    for s in rows:
        g = binding.varlen_attn_norm_fwd(flat[s], w, save="int8")
        assert torch.equal(f.out[s], g.out) and torch.equal(f.saved.codes[s], g.saved.codes) and torch.equal(f.rstd[s], g.rstd)
        assert torch.equal(dx[s], binding.varlen_attn_norm_bwd(flat[s], g.saved, g.mean, g.rstd, w)[0])
    total = sum(flat[a:a + 100_000].double().sum(0) for a in range(0, T, 100_000))
    size = sum(flat[a:a + 100_000].double().abs().sum(0) for a in range(0, T, 100_000))
    # a thread adds up T / (512 workgroups, 4 rows) rows, then 4 rows, then 512 / 32 and 32 partial sums: under 600 additions
    B.assert_within("db", db, total, 600 * B.U32 * size)
    del f, dx
    print("heads", flush=True)
    q = x[:, :12]
    wq = torch.rand(d, device="cuda")
    f = binding.varlen_attn_norm_fwd(q, wq)
    dx = binding.varlen_attn_norm_bwd(q, q, f.mean, f.rstd, wq)[0]
    for s in rows:
        g = binding.varlen_attn_norm_fwd(q[s], wq)
        assert torch.equal(f.out[s], g.out) and torch.equal(dx[s], binding.varlen_attn_norm_bwd(q[s], q[s], g.mean, g.rstd, wq)[0])


# What exceeds the last-level cache takes another form of the kernels: the same bits as a few of its rows by themselves.
@pytest.mark.parametrize("h,C,fmt", [(0, 64, "e4m3"), (0, 128, None), (0, 256, "int8"), (0, 512, "e4m3"), (0, 1024, "int8"), (0, 1280, "int8"),
                                     (0, 2048, "e4m3"), (0, 4096, "int8"), (0, 8192, None), (0, 16384, "int8"), (5, 64, None), (3, 320, "e4m3")])
def test_large_norms_give_the_bits_of_small_ones(h, C, fmt):
    from paper_2605_08962_amd import binding
    T = (1 << 27) // (C * max(h, 1)) + 3
    gen = torch.Generator(device="cuda").manual_seed(C)
    shape = (T, h, C) if h else (T, C)
    x, r, dy, ds = (torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(4))
    w, b = torch.rand(C, generator=gen, device="cuda"), torch.rand(C, generator=gen, device="cuda")

    def both(s):
        f = binding.varlen_attn_norm_fwd(x[s], w, b, residual=r[s], save=fmt)
        return [f.out, f.mean, f.rstd, f.summed, *(f.saved or ())], binding.varlen_attn_norm_bwd(dy[s], f.saved or f.summed, f.mean, f.rstd, w,
                                                                                                  dsummed=ds[s])
    whole, grads = both(slice(None))
    for s in (slice(0, 40), slice(T // 2, T // 2 + 40), slice(T - 40, T)):
        part, g = both(s)
        _same([t[s] for t in whole] + [grads[0][s]], part + [g[0]])
    mean, rstd = whole[1].double()[..., None], whole[2].double()[..., None]
    seen = B.act8_values(*whole[4:]) if fmt else whole[3]
    dw = (dy.double() * ((seen.double() - mean) * rstd))
    # a thread adds up at most T h / 512 rows (64 channels: 2^21 / 32768), then 32 row groups and 32 + 32 partial sums: under 400 additions
    B.assert_within("dw", grads[1], dw.flatten(0, -2).sum(0), 400 * B.U32 * dw.abs().flatten(0, -2).sum(0))
    B.assert_within("db", grads[2], dy.double().flatten(0, -2).sum(0), 400 * B.U32 * dy.double().abs().flatten(0, -2).sum(0))


@pytest.mark.parametrize("hq,hkv,d,P,interleaved", [(16, 16, 64, 32, False), (8, 2, 128, 64, False), (8, 8, 80, 40, False), (8, 4, 96, 48, True),
                                                    (8, 4, 128, 32, False), (4, 4, 80, 18, True), (3, 3, 66, 33, False)])
def test_large_rotations_and_packings_give_the_bits_of_small_ones(hq, hkv, d, P, interleaved):
    from paper_2605_08962_amd import binding
    T = (1 << 27) // ((hq + 2 * hkv) * d) + 5
    gen = torch.Generator(device="cuda").manual_seed(d)
    qkv = torch.randn((T, hq + 2 * hkv, d), generator=gen, device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 1 << 20, (2, T), generator=gen, device="cuda", dtype=torch.int32)
    freq, axis = torch.rand(P, generator=gen, device="cuda"), (torch.arange(P, device="cuda") % 2).int()

    def turn(x, pos, **kw):
        return binding.varlen_attn_rotary_fwd(x[:, :hq], x[:, hq:hq + hkv], pos, freq, axis, v=x[:, hq + hkv:], interleaved=interleaved, **kw)
    whole = turn(qkv, pos)
    packed = binding.varlen_attn_act8_pack(list(whole), "e4m3")
    back = binding.varlen_attn_act8_unpack(packed)
    for s in (slice(0, 40), slice(T // 2, T // 2 + 40), slice(T - 40, T)):
        part = turn(qkv[s], pos[:, s].contiguous())
        _same([t[s] for t in whole], list(part))
        p = binding.varlen_attn_act8_pack(list(part), "e4m3")
        _same([t[s] for x in packed for t in x], [t for x in p for t in x])
        _same([t[s] for t in back], binding.varlen_attn_act8_unpack(p))
    views = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    turn(qkv, pos, q_out=views[0], k_out=views[1], v_out=views[2])  # in place
    _same(list(whole), list(views))
