"""Weights held in 4 bits on the GPU, against the definition in 64 bits.

Tolerances.  A token's inputs enter as fixed-point numbers, off by 2^-26 of the token's largest at most; sums over a group are whole
numbers and exact.  With A = sum |w x| of an output: the four digits' sums of a group become fp32 numbers exactly, one fp32
FMA per group follows (at most K / 32), sums over at most 16 warps and 8 blocks, the join of the digits and two scalings:
(K / 32 + 16 + 8 + 8) * 2^-24 * A, and half a step of the output type.  A = sum over absolute digits' products may be twice sum |w x|
(a digit of the lower places has either sign): that doubles it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {0: torch.bfloat16, 1: torch.float32, 2: torch.float16}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pb():
    import __graft_entry__ as entry
    entry.build()
    from paper_2607_27591_b200 import binding
    return binding


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make_w4(seed, rows, cols, group, zeros, spread=1.0):
    g = gen(seed)
    n = -(-cols // group) if group else 1
    codes = torch.randint(0, 256, (rows, cols // 2), device="cuda", generator=g, dtype=torch.uint8)
    scales = (torch.rand(rows, n, device="cuda", generator=g) * 0.02 * spread + 1e-3).half()
    scales[::7] = 0                                              # groups without a weight
    z = torch.randint(0, 16, (rows, n), device="cuda", generator=g, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def values(w, group):
    codes, scales, zeros = w
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(1).double()
    width = group or q.shape[1]
    spread = lambda t: t.double().repeat_interleave(width, 1)[:, :q.shape[1]]
    return spread(scales) * (q - (8.0 if zeros is None else spread(zeros)))


def half_step(t, v):
    return torch.finfo(t).eps / 2 * v.abs() + torch.finfo(t).tiny * torch.finfo(t).eps


def sum_bound(K, A):
    return 2 * (K / 32 + 32) * U * A


def input_bound(x, W):
    """sum |w| 2^-26 max |x|, [B, N]"""
    return 2.0 ** -26 * x.abs().amax(1, keepdim=True) * W.abs().sum(1)


def tokens(seed, B, K, dtype):
    x = torch.randn(B, K, device="cuda", generator=gen(seed))
    x[:, ::97] *= 30
    return x.to(dtype)


def check_linear(y, w, group, x, K, ydt):
    W = values(w, group)
    xd = x.double()
    want = xd @ W.T
    tol = sum_bound(K, xd.abs() @ W.abs().T) + input_bound(xd, W)
    tol = tol + half_step(DT[ydt], want.abs() + tol)
    err = (y.double() - want).abs()
    assert torch.isfinite(y).all()
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))


LINEAR = [  # N, K, group, B, zeros, x type, y type
    (1, 32, 0, 1, False, 0, 1), (1, 32, 128, 1, True, 0, 0), (16, 32, 32, 1, False, 2, 2), (17, 64, 64, 2, True, 0, 1),
    (15, 96, 32, 7, True, 0, 1), (33, 160, 64, 8, False, 2, 1), (100, 224, 128, 9, True, 0, 1), (1024, 1024, 128, 1, False, 0, 0),
    (1024, 1024, 0, 3, True, 0, 1), (5003, 1376, 32, 3, True, 2, 2), (4096, 4096, 128, 8, False, 0, 1), (4097, 4096, 64, 5, True, 0, 0),
    (130, 14336, 128, 8, False, 0, 1), (4096, 14336, 128, 16, True, 0, 1), (64, 65536, 128, 16, False, 0, 1), (333, 4128, 128, 17, True, 0, 1),
    (300, 4096, 32, 33, False, 2, 1), (20011, 2048, 64, 1, True, 2, 1), (257, 8160, 0, 13, False, 0, 1), (2500, 512, 128, 1, True, 0, 1),
    (40, 320, 64, 4, True, 2, 1), (70, 1696, 32, 6, True, 0, 1), (3000, 192, 64, 2, False, 0, 1), (19, 12800, 0, 8, True, 0, 1), (2368, 16384, 64, 8, True, 0, 1),
]


@pytest.mark.parametrize("N,K,group,B,zeros,xdt,ydt", LINEAR)
def test_linear(pb, N, K, group, B, zeros, xdt, ydt):
    w = make_w4(N + K, N, K, group, zeros)
    x = tokens(N, B, K, DT[xdt])
    y = torch.full((B, N), float("nan"), dtype=DT[ydt], device="cuda")
    pb.prox_w4_linear(w, N, K, group, x, K, xdt, B, y, N, ydt)
    check_linear(y, w, group, x, K, ydt)
    again = torch.empty_like(y)
    pb.prox_w4_linear(w, N, K, group, x, K, xdt, B, again, N, ydt)
    assert torch.equal(y, again)


def test_linear_strides_and_alignment(pb):
    N, K, B = 1001, 1056, 5
    w = make_w4(3, N, K, 32, True)
    for offset, xs, ys in ((0, K + 8, N + 3), (1, K + 1, N), (3, K + 5, N + 1), (8, 2 * K, 2 * N)):
        flat = tokens(4, 1, offset + B * xs, torch.bfloat16)[0]
        x = flat[offset:].as_strided((B, K), (xs, 1))
        out = torch.full((B * ys + 7,), 5.0, device="cuda")
        y = out[1:].as_strided((B, N), (ys, 1))
        pb.prox_w4_linear(w, N, K, 32, flat[offset:], xs, 0, B, out[1:], ys, 1)
        check_linear(y, w, 32, x, K, 1)
        kept = torch.ones_like(out, dtype=torch.bool)
        kept[1:].as_strided((B, N), (ys, 1)).fill_(False)
        assert (out[kept] == 5.0).all()


def test_linear_tokens_do_not_meet(pb):
    """A token that is not finite spoils its own outputs only; the largest and smallest finite inputs are fine."""
    N, K, B = 272, 512, 6
    w = make_w4(5, N, K, 128, False, spread=0.01)
    x = tokens(6, B, K, torch.bfloat16)
    x[1] = float("inf")
    x[3, 7] = float("nan")
    x[4] *= 2.0 ** 100
    x[5] *= 2.0 ** -100
    y = torch.empty(B, N, device="cuda")
    pb.prox_w4_linear(w, N, K, 128, x, K, 0, B, y, N, 1)
    sane = [0, 2, 4, 5]
    check_linear(y[sane], w, 128, x[sane], K, 1)
    assert not torch.isfinite(y[1]).any() or (w[1][:, :] == 0).any()
    assert torch.isnan(y[3]).all()


def test_linear_far_rows(pb):
    """Rows behind 2^31 bytes of codes."""
    N, K = 140000, 32768
    codes = torch.randint(0, 256, (N, K // 2), device="cuda", generator=gen(1), dtype=torch.uint8)
    scales = torch.full((N, K // 128), 2.0 ** -8, device="cuda", dtype=torch.float16)
    x = tokens(2, 1, K, torch.bfloat16)
    y = torch.empty(1, N, device="cuda")
    pb.prox_w4_linear((codes, scales, None), N, K, 128, x, K, 0, 1, y, N, 1)
    assert N * K // 2 > 2 ** 31
    for part in (slice(0, 64), slice(N - 5000, N)):
        check_linear(y[:, part], (codes[part], scales[part], None), 128, x, K, 1)


def test_linear_streams_and_graphs(pb):
    N, K, B = 2048, 2048, 4
    w = make_w4(8, N, K, 64, True)
    x = tokens(9, B, K, torch.bfloat16)
    y = torch.empty(B, N, device="cuda")
    pb.prox_w4_linear(w, N, K, 64, x, K, 0, B, y, N, 1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y2 = torch.empty_like(y)
        pb.prox_w4_linear(w, N, K, 64, x, K, 0, B, y2, N, 1, side.cuda_stream)
    side.synchronize()
    assert torch.equal(y, y2)
    y3, y4 = torch.empty_like(y), torch.empty_like(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                                # the second call reads what the first has written (in bf16)
        s = torch.cuda.current_stream().cuda_stream
        pb.prox_w4_linear(w, N, K, 64, x, K, 0, B, y3, N, 1, s)
        xb = y3.to(torch.bfloat16)
        pb.prox_w4_linear(w, N, K, 64, xb, K, 0, B, y4, N, 1, s)
    x2 = tokens(10, B, K, torch.bfloat16)
    x.copy_(x2)
    graph.replay()
    torch.cuda.synchronize()
    check_linear(y3, w, 64, x2, K, 1)
    check_linear(y4, w, 64, y3.to(torch.bfloat16), K, 1)


def test_linear_chain_without_a_wait(pb):
    """Calls behind one another on a stream, each on the last one's output."""
    N = K = 1024
    ws = [make_w4(20 + i, N, K, 128, False) for i in range(6)]
    x = tokens(30, 2, K, torch.bfloat16)
    bufs = [x] + [torch.empty(2, N, dtype=torch.bfloat16, device="cuda") for _ in ws]
    for w, a, b in zip(ws, bufs, bufs[1:]):
        pb.prox_w4_linear(w, N, K, 128, a, K, 0, 2, b, N, 0)
    for w, a, b in zip(ws, bufs, bufs[1:]):
        check_linear(b, w, 128, a, K, 0)


def test_memory_that_a_kernel_cannot_read_is_refused(pb):
    """Pageable host memory in any place: refused on the host, nothing is launched."""
    N, K = 64, 128
    w = make_w4(12, N, K, 32, True)
    x, y = tokens(13, 1, K, torch.bfloat16), torch.empty(1, N, device="cuda")
    host = torch.zeros(1 << 16, dtype=torch.uint8)
    good = dict(w=w, x=x, y=y)
    for bad in (dict(w=(host, w[1], w[2])), dict(w=(w[0], host, w[2])), dict(w=(w[0], w[1], host)), dict(x=host), dict(y=host)):
        a = good | bad
        with pytest.raises(pb.ProxError) as e:
            pb.prox_w4_linear(a["w"], N, K, 32, a["x"], K, 0, 1, a["y"], N, 1)
        assert e.value.status == 1
    pb.prox_w4_linear(w, N, K, 32, x, K, 0, 1, y, N, 1)
    check_linear(y, w, 32, x, K, 1)


# ---- Stage 2 ----------------------------------------------------------------
def ffn_reference(gate, up, down, group, x, lists):
    """y and its bound: d(silu) <= 1.1 |dg|; expf, the division and the products lose a few steps; h s is rounded to fp32 and to a
    fixed-point number: 30 bits, less one, for the largest |h| times four times a scale, so off by 2^-27 of the largest |h| times the
    largest scale; a warp's sum of those is exact but for its shifts when a larger scale comes: half a unit each, and at most 20 of them
    (a shift is of 2 bits at least, fp16 has 40), in at most 128 warps; the sums of at most 16 warps and 8 blocks are fp32."""
    D = x.shape[1]
    ys, tols = [], []
    for b, ids in enumerate(lists):
        pick = lambda w: tuple(None if t is None else t[ids] for t in w)
        xd = x[b].double()
        G, Up, Dn = (values(pick(w), group) for w in (gate, up, down))
        g, u = G @ xd, Up @ xd
        dg = sum_bound(D, G.abs() @ xd.abs()) + input_bound(xd[None], G)[0]
        du = sum_bound(D, Up.abs() @ xd.abs()) + input_bound(xd[None], Up)[0]
        silu = g / (1 + torch.exp(-g))
        dsilu = 1.1 * dg + 16 * U * silu.abs() + 2.0 ** -126
        h = silu * u
        dh = dsilu * (u.abs() + du) + (silu.abs() + dsilu) * du + 4 * U * h.abs()
        y = h @ Dn
        A = (h.abs() + dh) @ Dn.abs()
        ys.append(y)
        most = (h.abs() + dh).max() * down[1].double().abs().max() if len(ids) else 0.0
        codes = (Dn / pick(down)[1].double().repeat_interleave(group or D, 1).clamp_min(1e-30)).abs().sum(0)
        tols.append(dh @ Dn.abs() + 2 * (16 + 8 + 8) * U * A + 2.0 ** -27 * most * codes + 20 * 128 * 2.0 ** -27 * most)
    return torch.stack(ys), torch.stack(tols)


def check_ffn(y, ref, ydt):
    want, tol = ref
    tol = tol + half_step(DT[ydt], want.abs() + tol)
    err = (y.double() - want).abs()
    assert torch.isfinite(y).all()
    assert (err <= tol).all(), (float((err / tol.clamp_min(1e-300)).max()), int((err > tol).sum()))


def ffn_case(seed, D, F, group, B, zeros):
    w = [make_w4(seed + i, F, D, group, zeros, spread=0.3) for i in range(3)]
    return (*w, tokens(seed + 5, B, D, torch.bfloat16))


def call_ffn(pb, case, D, F, group, B, sel, count, k2, ydt, stream=None):
    gate, up, down, x = case
    y = torch.full((B, D), float("nan"), dtype=DT[ydt], device="cuda")
    n = pb.prox_w4_stage2_workspace(D, F, B)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")      # whatever was in it
    pb.prox_w4_stage2_ffn(gate, up, down, D, F, group, x, B, sel, sel.stride(0), count, k2, y, ydt, ws, n, stream)
    return y


FFN = [  # D, F, k2, group, B, zeros, y type
    (128, 64, 1, 0, 1, False, 1), (128, 64, 64, 128, 8, True, 1), (512, 1536, 461, 0, 1, False, 1), (512, 1536, 461, 0, 3, True, 0),
    (384, 1000, 17, 128, 2, False, 1), (1024, 2752, 700, 128, 1, True, 1), (4096, 12288, 2867, 128, 1, False, 1), (4096, 12288, 2867, 128, 4, False, 0),
    (8192, 2048, 512, 128, 8, True, 1), (16384, 704, 350, 128, 8, False, 1), (16384, 704, 9, 0, 1, True, 1), (640, 65536, 6000, 128, 2, False, 1),
    (2048, 5504, 5504, 0, 5, False, 1), (1152, 3008, 1203, 128, 6, False, 1), (256, 333, 100, 128, 7, True, 1),
    (384, 1000, 200, 128, 3, True, 1), (1152, 640, 333, 128, 8, True, 0), (640, 2000, 1999, 0, 2, True, 1), (16384, 1024, 900, 128, 7, True, 1), (128, 65536, 65536, 128, 1, True, 1),
]


@pytest.mark.parametrize("D,F,k2,group,B,zeros,ydt", FFN)
def test_ffn(pb, D, F, k2, group, B, zeros, ydt):
    case = ffn_case(D + F, D, F, group, B, zeros)
    sel = torch.rand(B, F, device="cuda", generator=gen(k2)).argsort(1)[:, :k2].sort(1).values.to(torch.int32).contiguous()
    y = call_ffn(pb, case, D, F, group, B, sel, None, k2, ydt)
    check_ffn(y, ffn_reference(*case[:3], group, case[3], [sel[b].long() for b in range(B)]), ydt)
    assert torch.equal(y, call_ffn(pb, case, D, F, group, B, sel, None, k2, ydt))


@pytest.mark.parametrize("B", [1, 2, 5, 8])
def test_ffn_counts_and_bad_ids(pb, B):
    """Lists of different lengths (none, one, all, more than all), in any order, with ids that are no channels."""
    D, F, k2, group = 512, 1408, 300, 128
    case = ffn_case(70 + B, D, F, group, B, B == 5)
    sel = torch.rand(B, F, device="cuda", generator=gen(B)).argsort(1)[:, :k2].to(torch.int32)
    sel[:, 5], sel[:, 11], sel[:, 200] = -1, F, 2 ** 31 - 1
    wide = torch.full((B, k2 + 13), -7, dtype=torch.int32, device="cuda")
    wide[:, :k2] = sel
    for counts in ([0] * B, [1] * B, [[0, 300, 7, 1, 299, 16, 150, 300][(b + B) % 8] for b in range(B)], [1000] * B, [-3] * B):
        count = torch.tensor(counts, dtype=torch.int32, device="cuda")
        y = call_ffn(pb, case, D, F, group, B, wide, count, k2, 1)
        lists = []
        for b in range(B):
            ids = sel[b, :max(0, min(k2, counts[b]))].long()
            lists.append(ids[(ids >= 0) & (ids < F)])
        check_ffn(y, ffn_reference(*case[:3], group, case[3], lists), 1)
    y = call_ffn(pb, case, D, F, group, B, wide, None, 0, 1)
    assert (y == 0).all()


def test_ffn_batch_rows_stand_alone(pb):
    """A token's result is the one that it gets alone, whatever its neighbours hold."""
    D, F, k2, B = 1024, 2816, 900, 8
    case = ffn_case(90, D, F, 128, B, False)
    sel = torch.rand(B, F, device="cuda", generator=gen(91)).argsort(1)[:, :k2].sort(1).values.to(torch.int32).contiguous()
    case[3][2] = float("nan")
    y = call_ffn(pb, case, D, F, 128, B, sel, None, k2, 1)
    good = [b for b in range(B) if b != 2]
    ref = ffn_reference(*case[:3], 128, case[3][good], [sel[b].long() for b in good])
    check_ffn(y[good], ref, 1)
    assert torch.isnan(y[2]).all()


def test_ffn_scales_that_rise(pb):
    """Scales of the down projection that grow along the list by 2^20, and a long run of zero scales before them."""
    D, F, B = 256, 4096, 2
    gate, up, down, x = ffn_case(93, D, F, 128, B, True)
    scale = torch.exp2(torch.arange(F, device="cuda") / 200.0 - 18)[:, None].expand(F, 2).clone()
    scale[:1000] = 0
    down = (down[0], scale.half(), down[2])
    sel = torch.arange(F, dtype=torch.int32, device="cuda").expand(B, F).contiguous()
    case = (gate, up, down, x)
    for n in (F, 2500, 1200, 900):
        y = call_ffn(pb, case, D, F, 128, B, sel, None, n, 1)
        check_ffn(y, ffn_reference(gate, up, down, 128, x, [sel[b, :n].long() for b in range(B)]), 1)


def test_ffn_graphs_with_a_workspace_each(pb):
    D, F, k2, B, group = 512, 1536, 400, 3, 128
    case = ffn_case(95, D, F, group, B, False)
    sel = torch.rand(B, F, device="cuda", generator=gen(96)).argsort(1)[:, :k2].sort(1).values.to(torch.int32).contiguous()
    n = pb.prox_w4_stage2_workspace(D, F, B)
    outs, graphs = [], []
    for i in range(2):
        y, ws = torch.empty(B, D, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda")
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            pb.prox_w4_stage2_ffn(*case[:3], D, F, group, case[3], B, sel, k2, None, k2, y, 1, ws, n, torch.cuda.current_stream().cuda_stream)
        outs.append((y, ws)); graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    ref = ffn_reference(*case[:3], group, case[3], [sel[b].long() for b in range(B)])
    for y, _ in outs:
        check_ffn(y, ref, 1)


def test_ffn_behind_the_mask_of_stage_1(pb):
    """prox_stage1_mask and then Stage 2 over 4-bit weights, top-k and threshold form; the 4-bit matrices from prox_w4_quantize."""
    from paper_2607_27591_b200 import inputs
    wl, wg, wu, wd, x = inputs.make_workload("toy", n_tokens=4)
    D, F = wl.d_model, wl.d_ff
    k1, k2 = wl.points[50]
    dev = lambda bits: torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    tg, tu, td, tx = dev(wg), dev(wu), dev(wd), dev(x)
    w4 = []
    for w in (tg, tu, td.t().contiguous()):
        codes, scales = torch.empty(F, D // 2, dtype=torch.uint8, device="cuda"), torch.empty(F, D // 128, dtype=torch.float16, device="cuda")
        pb.prox_w4_quantize(w, F, D, 128, codes, scales)
        w4.append((codes, scales, None))
    h = pb.prox_ffn_create(D, F, 4, 1, tg, tu, td)
    try:
        pb.prox_quantize_proxy(h, 4, 128)
        sel = torch.empty(4, k2, dtype=torch.int32, device="cuda")
        pb.prox_stage1_mask(h, tx, 4, k1, k2, sel)
        y = call_ffn(pb, (*w4, tx), D, F, 128, 4, sel, None, k2, 1)
        check_ffn(y, ffn_reference(*w4, 128, tx, [sel[b].long() for b in range(4)]), 1)
        exact = torch.empty(4, D, device="cuda")
        pb.prox_stage2_ffn(h, tx, 4, sel, k2, exact)
        assert float((y - exact).norm() / exact.norm()) < 0.35     # weights off by 0.11 of their deviation (a step of 2.7 / 7, over sqrt 12), three factors: 0.2; SiLU's slope adds to one
        sel, count = torch.empty(4, F, dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
        pb.prox_stage1_mask_threshold(h, tx, 4, 0.5, 0.2, sel, count)
        y = call_ffn(pb, (*w4, tx), D, F, 128, 4, sel, count, F, 1)
        n = count.tolist()
        check_ffn(y, ffn_reference(*w4, 128, tx, [sel[b, :n[b]].long() for b in range(4)]), 1)
    finally:
        pb.prox_ffn_destroy(h)


# ---- packer -----------------------------------------------------------------
@pytest.mark.parametrize("rows,cols,group", [(1, 32, 0), (7, 96, 32), (64, 160, 64), (33, 288, 128), (100, 4096, 128), (5, 8192, 0)])
def test_quantize_is_the_rule_of_the_proxies(pb, rows, cols, group):
    from oracle import prox_oracle as po
    w = (torch.randn(rows, cols, device="cuda", generator=gen(rows)) * 0.02).bfloat16()
    w[0, : min(cols, 32)] = 0
    width = group or cols
    pad = (-cols) % width
    q, s = po.quantize_proxy(torch.nn.functional.pad(w.float(), (0, pad)).cpu().numpy(), 4, group)
    n = (cols + width - 1) // width
    codes = torch.full((rows, cols // 2), 255, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, n, dtype=torch.float16, device="cuda")
    pb.prox_w4_quantize(w, rows, cols, group, codes, scales)
    got = torch.stack((codes & 15, codes >> 4), -1).flatten(1).cpu().numpy().astype(np.int8) - 8
    assert np.array_equal(got, q[:, :cols])
    assert np.array_equal(scales.cpu().numpy().reshape(rows, n), np.asarray(s).reshape(rows, n))
