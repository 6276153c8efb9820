"""prox_token_logprobs on the GPU, against log_softmax in 64 bits.

Tolerances (d = z - max z, p = softmax).  Every d is a difference, rounded, times a rounded factor: off by 3 steps of 2^-24 |d|.  An
exponential has the approximation's 2^-22 and what d is off: s by sum p (2^-22 + 3 2^-24 |d|), w by sum p |d| of the same; sums of a thread
(16 a round, V / 16384 rounds), 5 + 4 + 3 joins of two roundings and an exponential each: (V / 1024 + 64) 2^-24 more.  log p adds its own
difference, product and subtraction, the logarithm 2 steps."""
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


def call(pb, x, dt, V, temperature, given, top, entropy=True, stream=None):
    T, n = x.shape[0], 0 if given is None else given.shape[1]
    lp = torch.full((T, n), 7.0, device="cuda")
    en = torch.full((T,), 7.0, device="cuda") if entropy else None
    tl, ti = torch.full((T, top), 7.0, device="cuda"), torch.full((T, top), -7, dtype=torch.int32, device="cuda")
    pb.prox_token_logprobs(x, dt, T, V, x.stride(0), temperature, given, n, lp, en, top, tl, ti, stream)
    return lp, en, tl, ti


def check(x, V, temperature, given, top, out):
    """Rows with finite maxima."""
    lp, en, tl, ti = out
    z = x.double() / temperature
    m = z.amax(1, keepdim=True)
    d = z - m
    p = torch.softmax(z, 1)
    logp = torch.log_softmax(z, 1)
    dd = torch.where(p > 0, d.abs(), 0.0)
    e1, e2 = (p * dd).sum(1), (p * dd * dd).sum(1)
    sums = (V / 1024 + 64) * U
    tol_s = 4 * U + 3 * U * e1 + sums
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(1)
    if en is not None:
        tol = tol_s * 2 + 4 * U * e1 + 3 * U * e2 + sums * e1 + 4 * U * (entropy.abs() + e1) + 1e-7
        assert ((en.double() - entropy).abs() <= tol).all(), float(((en.double() - entropy).abs() / tol).max())

    def close(got, index):
        want = logp.gather(1, index)
        far = d.gather(1, index).abs()
        fine = torch.isfinite(want)
        assert (got[~fine].double() == want[~fine]).all()
        tol = tol_s[:, None] + 4 * U * far + 4 * U * want.abs() + 4 * U * logp.amax(1).abs()[:, None]
        err = (got.double() - want).abs()
        assert (err[fine] <= tol[fine]).all(), float((err[fine] / tol[fine]).max())

    if given is not None and given.numel():
        close(lp, given.long())
    if top:
        order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(ti.long(), order)
        close(tl, order)


CASES = [  # T, V, type, given, top, temperature, extra stride
    (1, 1, 0, 1, 1, 1.0, 0), (3, 2, 1, 2, 2, 0.5, 1), (5, 31, 2, 3, 31, 1.0, 0), (7, 32, 0, 1, 32, 1.0, 5), (4, 33, 0, 1, 32, 2.0, 0),
    (1, 131072, 0, 1, 20, 1.0, 0), (1, 131073, 0, 2, 32, 1.0, 0), (2, 50001, 1, 4, 5, 0.7, 3), (37, 50001, 1, 4, 5, 0.7, 3), (37, 50001, 0, 4, 5, 1.3, 3),
    (160, 32000, 0, 1, 20, 1.0, 0), (300, 4099, 2, 1, 1, 1.0, 1), (2000, 1000, 0, 1, 3, 1.0, 0), (9, 262144, 1, 1, 32, 1.0, 0), (3, 1000003, 0, 5, 32, 1.0, 1),
    (40, 16385, 0, 700, 0, 1.0, 7), (64, 8191, 2, 0, 8, 0.9, 0), (150, 131072, 0, 1, 0, 1.0, 0),
]


@pytest.mark.parametrize("T,V,dt,given,top,temperature,pad", CASES)
def test_rows(pb, T, V, dt, given, top, temperature, pad):
    g = gen(T + V)
    flat = torch.randn(T, V + pad, device="cuda", generator=g) * 3
    flat += torch.empty_like(flat).exponential_(1.0, generator=g)
    x = flat.to(DT[dt])[:, :V]
    ids = torch.randint(0, V, (T, given), device="cuda", generator=g, dtype=torch.int32) if given else None
    out = call(pb, x, dt, V, temperature, ids, top)
    check(x, V, temperature, ids, top, out)
    again = call(pb, x, dt, V, temperature, ids, top)
    for a, b in zip(out, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", [0, 1, 2])
def test_orders_that_fill_the_list(pb, dt):
    """Rising, falling and equal logits, steps with many equal ones, large ones all in one thread's vectors or in one stretch."""
    V, top = 70001, 32
    i = torch.arange(V, device="cuda", dtype=torch.float32)
    rows = [i / 2000, -i / 2000, torch.zeros(V, device="cuda"), torch.floor(i / 300) / 20, torch.floor(-i / 9000), (i % 512 == 5).float() * 9 + i * 1e-4,
            ((i > 30000) & (i < 40000)).float() * 5, (i == V - 1).float(), -(i % 7), torch.where(i % 4096 < 32, 10.0 + i / 70001, -i / 70001)]
    x = torch.stack(rows).to(DT[dt])
    ids = torch.tensor([[0], [V - 1]] * 5, dtype=torch.int32, device="cuda")
    check(x, V, 1.0, ids, top, call(pb, x, dt, V, 1.0, ids, top))
    # the same a row at a time: split over blocks
    for r in range(len(rows)):
        check(x[r:r + 1], V, 1.0, ids[r:r + 1], top, call(pb, x[r:r + 1], dt, V, 1.0, ids[r:r + 1], top))
    # ... and in one block each (rows enough to fill the GPU)
    many = x[torch.arange(200, device="cuda") % len(rows)].contiguous()
    out = call(pb, many, dt, V, 1.0, None, top)
    want = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(out[3].long(), want[torch.arange(200, device="cuda") % len(rows)])


@pytest.mark.parametrize("dt", [0, 1, 2])
@pytest.mark.parametrize("T", [6, 400])
def test_masks(pb, dt, T):
    """Most logits -inf or the type's lowest value; rows of nothing else."""
    V, top, g = 9001, 8, gen(dt + T)
    low = torch.finfo(DT[dt]).min
    x = (torch.randn(T, V, device="cuda", generator=g) * 4).to(DT[dt])
    masked = torch.rand(T, V, device="cuda", generator=g) < 0.95
    x[0::3] = x[0::3].masked_fill(masked[0::3], float("-inf"))
    x[1::3] = x[1::3].masked_fill(masked[1::3], low)
    x[2] = float("-inf")
    x[3] = low
    x[4] = float("-inf")
    x[4, V - 1] = low
    x[5] = float("-inf")
    x[5, :9] = low
    ids = torch.randint(0, V, (T, 3), device="cuda", generator=g, dtype=torch.int32)
    lp, en, tl, ti = call(pb, x, dt, V, 1.0, ids, top)
    some = torch.ones(T, dtype=torch.bool, device="cuda")
    some[2] = False
    check(x[some], V, 1.0, ids[some], top, (lp[some], en[some], tl[some], ti[some]))
    assert torch.isneginf(lp[2]).all() and en[2] == 0 and torch.isneginf(tl[2]).all()
    assert ti[2].tolist() == list(range(top))


@pytest.mark.parametrize("dt", [0, 1, 2])
@pytest.mark.parametrize("T", [4, 300])
def test_what_is_not_finite_stays_in_its_row(pb, dt, T):
    V, top, g = 20000, 5, gen(40 + dt)
    x = (torch.randn(T, V, device="cuda", generator=g) * 2).to(DT[dt])
    x[1, 777] = float("nan")
    x[1, 19999] = float("nan")
    x[2, 5000] = float("inf")
    ids = torch.randint(0, V, (T, 2), device="cuda", generator=g, dtype=torch.int32)
    lp, en, tl, ti = call(pb, x, dt, V, 1.0, ids, top)
    rest = [r for r in range(T) if r not in (1, 2)]
    check(x[rest], V, 1.0, ids[rest], top, (lp[rest], en[rest], tl[rest], ti[rest]))
    for r in (1, 2):
        assert torch.isnan(lp[r]).all() and torch.isnan(en[r]) and torch.isnan(tl[r]).all()
    assert ti[1, :2].tolist() == [777, 19999] and ti[2, 0] == 5000


def test_signed_zeros_are_equal(pb):
    x = torch.full((1, 100), -1.0, device="cuda")
    x[0, 10], x[0, 20], x[0, 30] = -0.0, 0.0, -0.0
    assert call(pb, x, 1, 100, 1.0, None, 4)[3][0].tolist() == [10, 20, 30, 0]


def test_ids_that_are_no_tokens(pb):
    V = 1000
    x = torch.randn(3, V, device="cuda", generator=gen(1))
    ids = torch.tensor([[-1, 5, V], [-100, V - 1, 2 ** 31 - 1], [0, -(2 ** 31), 1]], dtype=torch.int32, device="cuda")
    lp = call(pb, x, 1, V, 1.0, ids, 0)[0]
    assert lp[0, 0] == 0 and lp[1, 0] == 0 and lp[2, 1] == 0
    assert torch.isnan(lp[0, 2]) and torch.isnan(lp[1, 2])
    want = torch.log_softmax(x.double(), 1)
    for r, c, v in ((0, 1, 5), (1, 1, V - 1), (2, 0, 0), (2, 2, 1)):
        assert abs(float(lp[r, c]) - float(want[r, v])) < 1e-5


def test_parts_can_be_left_out(pb):
    V = 5000
    x = torch.randn(2, V, device="cuda", generator=gen(2))
    ids = torch.tensor([[3], [4]], dtype=torch.int32, device="cuda")
    full = call(pb, x, 1, V, 1.0, ids, 6)
    lp = torch.empty(2, 1, device="cuda")
    pb.prox_token_logprobs(x, 1, 2, V, V, 1.0, ids, 1, lp, None, 0, None, None)
    en = torch.empty(2, device="cuda")
    pb.prox_token_logprobs(x, 1, 2, V, V, 1.0, None, 0, None, en, 0, None, None)
    tl, ti = torch.empty(2, 6, device="cuda"), torch.empty(2, 6, dtype=torch.int32, device="cuda")
    pb.prox_token_logprobs(x, 1, 2, V, V, 1.0, None, 0, None, None, 6, tl, ti)
    for a, b in zip(full, (lp, en, tl, ti)):
        assert torch.equal(a, b)


def test_unaligned_rows_of_16_bits(pb):
    V, T = 3001, 11
    flat = torch.randn(T * V + 9, device="cuda", generator=gen(3)).bfloat16()
    for offset in (0, 1, 3, 7):
        x = flat[offset:offset + T * V].view(T, V)
        ids = torch.arange(T, device="cuda", dtype=torch.int32)[:, None] * 200
        check(x, V, 1.0, ids, 9, call(pb, x, 0, V, 1.0, ids, 9))


@pytest.mark.parametrize("temperature", [1e-3, 0.05, 30.0, 1e6])
def test_temperatures(pb, temperature):
    V = 40000
    x = torch.randn(5, V, device="cuda", generator=gen(4)) * 3
    ids = torch.randint(0, V, (5, 4), device="cuda", generator=gen(5), dtype=torch.int32)
    check(x, V, temperature, ids, 4, call(pb, x, 1, V, temperature, ids, 4))


def test_far_rows(pb):
    """Rows behind 2^32 bytes."""
    V, T = 300001, 7400
    x = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    for r in range(0, T, 500):
        x[r:r + 500].normal_(0.0, 2.0, generator=gen(r))
    ids = torch.randint(0, V, (T, 1), device="cuda", generator=gen(6), dtype=torch.int32)
    assert T * V * 2 > 2 ** 32
    lp, en, tl, ti = call(pb, x, 0, V, 1.0, ids, 2)
    for part in (slice(0, 4), slice(T - 8, T)):
        check(x[part], V, 1.0, ids[part], 2, (lp[part], en[part], tl[part], ti[part]))


def test_streams_and_graphs(pb):
    V, T, top = 50000, 6, 10
    x = torch.randn(T, V, device="cuda", generator=gen(7))
    ids = torch.randint(0, V, (T, 2), device="cuda", generator=gen(8), dtype=torch.int32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out = call(pb, x, 1, V, 1.0, ids, top, stream=side.cuda_stream)
    side.synchronize()
    check(x, V, 1.0, ids, top, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = x * 2
        out = call(pb, y, 1, V, 1.0, ids, top, stream=torch.cuda.current_stream().cuda_stream)
    x.copy_(torch.randn(T, V, device="cuda", generator=gen(9)))
    graph.replay()
    torch.cuda.synchronize()
    check(x * 2, V, 1.0, ids, top, out)


def test_a_decode_step_with_its_log_probabilities(pb):
    """Stage-1 mask, Stage 2 over 4-bit weights, residual, norm, a 4-bit head and the log probabilities of its logits: every step is
    checked on what the library handed on to it."""
    from paper_2607_27591_b200 import inputs
    from tests.test_gpu_w4 import check_ffn, check_linear, ffn_reference
    wl, wg, wu, wd, x = inputs.make_workload("toy", n_tokens=3)
    D, F, V, B = wl.d_model, wl.d_ff, 5003, 3
    k1, k2 = wl.points[50]
    dev = lambda bits: torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    tg, tu, td, tx = dev(wg), dev(wu), dev(wd), dev(x)

    def pack(w, group):
        rows, cols = w.shape
        codes, scales = torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda"), torch.empty(rows, cols // group, dtype=torch.float16, device="cuda")
        pb.prox_w4_quantize(w, rows, cols, group, codes, scales)
        return codes, scales, None

    w4 = [pack(tg, 128), pack(tu, 128), pack(td.t().contiguous(), 128)]
    head = pack((torch.randn(V, D, device="cuda", generator=gen(11)) * 0.05).bfloat16(), 64)
    s = torch.cuda.current_stream().cuda_stream
    h = pb.prox_ffn_create(D, F, B, 1, tg, tu, td, s)
    try:
        pb.prox_quantize_proxy(h, 4, 128, s)
        sel = torch.empty(B, k2, dtype=torch.int32, device="cuda")
        pb.prox_stage1_mask(h, tx, B, k1, k2, sel, None, s)
        n = pb.prox_w4_stage2_workspace(D, F, B)
        ws, y = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(B, D, device="cuda")
        pb.prox_w4_stage2_ffn(*w4, D, F, 128, tx, B, sel, k2, None, k2, y, 1, ws, n, s)
        res = tx.float() + y
        norm_w, xn = torch.ones(D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, D, dtype=torch.bfloat16, device="cuda")
        pb.prox_rmsnorm(h, res, norm_w, 1e-6, B, xn, s)
        logits = torch.empty(B, V, device="cuda")
        pb.prox_w4_linear(head, V, D, 64, xn, D, 0, B, logits, V, 1, s)
        ids = torch.tensor([[1], [V - 1], [77]], dtype=torch.int32, device="cuda")
        out = call(pb, logits, 1, V, 1.0, ids, 20, stream=s)
        torch.cuda.synchronize()
        check_ffn(y, ffn_reference(*w4, 128, tx, [sel[b].long() for b in range(B)]), 1)
        check_linear(logits, head, 64, xn, D, 1)
        check(logits, V, 1.0, ids, 20, out)
    finally:
        pb.prox_ffn_destroy(h)
