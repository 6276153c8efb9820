"""Weights held in 4 bits at the edges of what the calls allow, against the definition in 64 bits.  Tolerances: those of
tests/test_gpu_w4.py, and for the down projection a narrower one (own_reference)."""
import pytest
import torch

from tests.test_gpu_w4 import U, call_ffn, check_ffn, check_linear, ffn_case, ffn_reference, gen, input_bound, make_w4, sum_bound, tokens, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pb():
    import __graft_entry__ as entry
    entry.build()
    from paper_2607_27591_b200 import binding
    return binding


@pytest.mark.parametrize("K", [12288, 12320, 12416, 12544, 12576])
@pytest.mark.parametrize("B", [6, 7, 8, 16, 19])
def test_linear_rows_between_four_blocks_and_eight(pb, K, B):
    """Groups of 32: for 7 and 8 tokens K = 12320 .. 12544 fits in neither a cluster of four nor one of eight."""
    N, group = 130, 32
    w = make_w4(K + B, N, K, group, B == 8)
    x = tokens(B, B, K, torch.bfloat16)
    y = torch.full((B, N), float("nan"), device="cuda")
    pb.prox_w4_linear(w, N, K, group, x, K, 0, B, y, N, 1)
    check_linear(y, w, group, x, K, 1)


def lists(seed, B, F, k2):
    return torch.rand(B, F, device="cuda", generator=gen(seed)).argsort(1)[:, :k2].sort(1).values.to(torch.int32).contiguous()


@pytest.mark.parametrize("powers", [[-55], [-60], [58], [-58, 0, 55], [-52, -60, 58, 3, -45]])
@pytest.mark.parametrize("zeros", [False, True])
def test_ffn_small_and_large_inputs(pb, powers, zeros):
    """h goes with the square of the inputs: from near the least to near the largest number of fp32.  (Inputs of one size a token; y stays
    a normal number, so the bound is as tight as for inputs near 1.)"""
    D, F, k2, B = 512, 1408, 500, len(powers)
    gate, up, down, x = ffn_case(300 + B, D, F, 128, B, zeros)
    x = (x.float() * torch.exp2(torch.tensor(powers, device="cuda", dtype=torch.float32))[:, None]).bfloat16()
    sel = lists(301, B, F, k2)
    y = call_ffn(pb, (gate, up, down, x), D, F, 128, B, sel, None, k2, 1)
    ref = ffn_reference(gate, up, down, 128, x, [sel[b].long() for b in range(B)])
    assert (ref[0].abs().amax(1) > 2.0 ** -126).all()
    check_ffn(y, ref, 1)


def own_reference(gate, up, down, group, x, kept):
    """y and a bound in which nothing but a token's own channels counts.  As ffn_reference, but the fixed-point numbers h s are off by
    2^-24 of the largest |h s| that the token has in the column's group: when the exponent is set, that one takes at least 2^23 of 2^30
    (6 bits are kept free above it, and an exponent is a whole number), and rounding is off by half a unit.  When the exponent
    falls, by 3 bits at least, a sum of codes and one of zero points are rounded by half a unit each: 8/7 units of 2^-23 in all, in
    each of at most 128 warps: 300 times 2^-24."""
    D = x.shape[1]
    ys, tols = [], []
    for b, ids in enumerate(kept):
        pick = lambda w: tuple(None if t is None else t[ids] for t in w)
        xd = x[b].double()
        G, Up, Dn = (values(pick(w), group) for w in (gate, up, down))
        s = pick(down)[1].double().repeat_interleave(group or D, 1)[:, :D]
        g, u = G @ xd, Up @ xd
        dg = sum_bound(D, G.abs() @ xd.abs()) + input_bound(xd[None], G)[0]
        du = sum_bound(D, Up.abs() @ xd.abs()) + input_bound(xd[None], Up)[0]
        silu = g / (1 + torch.exp(-g))
        dsilu = 1.1 * dg + 16 * U * silu.abs() + 2.0 ** -126
        h = silu * u
        dh = dsilu * (u.abs() + du) + (silu.abs() + dsilu) * du + 4 * U * h.abs()
        A = (h.abs() + dh) @ Dn.abs()
        most = ((h.abs() + dh)[:, None] * s).amax(0)
        codes = (Dn / s.clamp_min(1e-30)).abs().sum(0)
        ys.append(h @ Dn)
        tols.append(dh @ Dn.abs() + 2 * (16 + 8 + 8) * U * A + 2.0 ** -24 * most * (codes + 300))
    return torch.stack(ys), torch.stack(tols)


def with_scales(w, rows, factor):
    """w with the scales of some rows multiplied (and held to what fp16 has)."""
    scales = w[1].clone()
    scales[rows] = (scales[rows].float() * factor).clamp(max=65504).half()
    return w[0], scales, w[2]


def with_scale(w, rows, scale):
    scales = w[1].clone()
    scales[rows] = scale
    return w[0], scales, w[2]


@pytest.mark.parametrize("B", [2, 3, 6, 8])
@pytest.mark.parametrize("zeros", [False, True])
def test_ffn_channels_of_other_tokens_do_not_count(pb, B, zeros):
    """Channels that the last token alone keeps have scales up to 2^22 times larger in the down projection: the other tokens' results
    are as exact as without them."""
    D, F, k2, group = 512, 1408, 300, 128
    gate, up, down, x = ffn_case(400 + B, D, F, group, B, zeros)
    sel = lists(401, B, F, k2)
    others = torch.zeros(F, dtype=torch.bool, device="cuda")
    others[sel[:-1].flatten().long()] = True
    alone = sel[-1][~others[sel[-1].long()]].long()
    assert len(alone) > 20
    for factor in (2.0 ** 12, 2.0 ** 22):
        big = with_scales(down, alone, factor)
        y = call_ffn(pb, (gate, up, big, x), D, F, group, B, sel, None, k2, 1)
        check_ffn(y, own_reference(gate, up, big, group, x, [sel[b].long() for b in range(B)]), 1)


@pytest.mark.parametrize("zeros", [False, True])
def test_ffn_skipped_ids_do_not_count(pb, zeros):
    """Ids that are no channels, in every tile of the list, while channel 0 (which is in no list) has the largest scale that there is."""
    D, F, k2, group = 512, 1408, 400, 128
    for B in (1, 4):
        gate, up, down, x = ffn_case(410 + B, D, F, group, B, zeros)
        down = with_scale(down, [0], 65504.0)
        sel = lists(411, B, F - 1, k2) + 1
        sel[:, ::9], sel[:, 3::31] = -1, F
        y = call_ffn(pb, (gate, up, down, x), D, F, group, B, sel, None, k2, 1)
        kept = [sel[b][(sel[b] >= 0) & (sel[b] < F)].long() for b in range(B)]
        check_ffn(y, own_reference(gate, up, down, group, x, kept), 1)


@pytest.mark.parametrize("B", [1, 5])
@pytest.mark.parametrize("group", [0, 128])
def test_ffn_large_h_with_a_small_scale(pb, B, group):
    """Channels whose h is some 2^28 times larger and whose scales in the down projection are 0, and channels whose h is as much larger as
    their scales are smaller: products, not the largest h times the largest scale, set the precision."""
    D, F, k2 = 512, 1408, 600
    gate, up, down, x = ffn_case(420 + B, D, F, group, B, False)
    loud, quiet = torch.arange(5, F, 97, device="cuda"), torch.arange(11, F, 101, device="cuda")
    gate = with_scales(gate, loud, 2.0 ** 8)
    up = with_scales(with_scales(up, loud, 2.0 ** 20), quiet, 2.0 ** 14)
    down = with_scales(with_scale(down, loud, 0.0), quiet, 2.0 ** -14)
    sel = lists(421, B, F, k2)
    y = call_ffn(pb, (gate, up, down, x), D, F, group, B, sel, None, k2, 1)
    check_ffn(y, own_reference(gate, up, down, group, x, [sel[b].long() for b in range(B)]), 1)


@pytest.mark.parametrize("B", [1, 2, 8])
def test_ffn_products_that_rise_and_fall(pb, B):
    """Scales of the down projection that grow by 2^30 along the list, fall again, and are 0 for long runs."""
    D, F, group = 256, 6144, 128
    gate, up, down, x = ffn_case(430 + B, D, F, group, B, True)
    j = torch.arange(F, device="cuda")
    for power in (j / 200.0 - 20, 10 - j / 200.0, (j % 640) / 25.0 - 15):
        scale = torch.exp2(power.float())[:, None].expand(F, 2).clone()
        scale[1000:2000] = 0
        big = (down[0], scale.half(), down[2])
        sel = j.to(torch.int32).expand(B, F).contiguous()
        y = call_ffn(pb, (gate, up, big, x), D, F, group, B, sel, None, F, 1)
        check_ffn(y, own_reference(gate, up, big, group, x, [sel[b].long() for b in range(B)]), 1)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("B", [1, 2, 3, 8])
def test_ffn_a_scale_that_is_not_finite_stays_with_its_tokens(pb, B, bad):
    """A scale of the down projection that is not finite makes NaN of the outputs of its column group, for the tokens that keep its channel;
    no other output changes.  In a channel of one token, in one of all, and in channel 0 where it stands for skipped ids."""
    D, F, k2, group = 512, 1408, 300, 128
    gate, up, down, x = ffn_case(440 + B, D, F, group, B, B == 3)
    sel = lists(441, B, F - 1, k2) + 1
    sel[:, 7] = -1                                               # ids that are skipped
    kept = [sel[b][sel[b] >= 0].long() for b in range(B)]
    plain = call_ffn(pb, (gate, up, down, x), D, F, group, B, sel, None, k2, 1)
    check_ffn(plain, own_reference(gate, up, down, group, x, kept), 1)
    some = [ids[ids % 7 != 0] for ids in kept]                   # (of every seventh channel the gate's scales are 0, and so is h)
    for channel in (0, int(some[-1][100]), int(some[0][-1])):
        broken = with_scale(down, (channel, 2), bad)
        y = call_ffn(pb, (gate, up, broken, x), D, F, group, B, sel, None, k2, 1)
        ref, tol = own_reference(gate, up, down, group, x, kept)
        for b in range(B):
            hit = bool((kept[b] == channel).any())
            assert torch.isnan(y[b, 256:384]).all() == hit, (channel, b)
            rest = torch.cat((torch.arange(256), torch.arange(384 if hit else 256, D)))
            check_ffn(y[b:b + 1, rest], (ref[b:b + 1, rest], tol[b:b + 1, rest]), 1)


@pytest.mark.parametrize("B", [1, 4])
def test_ffn_a_gate_scale_that_is_not_finite_stays_with_its_tokens(pb, B):
    D, F, k2, group = 512, 1408, 300, 128
    gate, up, down, x = ffn_case(450 + B, D, F, group, B, False)
    sel = lists(451, B, F, k2)
    channel = int(sel[-1][sel[-1] % 7 != 0][9])
    for w in (0, 1):
        m = [gate, up]
        m[w] = with_scale(m[w], (channel, 1), float("inf"))
        y = call_ffn(pb, (*m, down, x), D, F, group, B, sel, None, k2, 1)
        for b in range(B):
            if bool((sel[b] == channel).any()):
                assert not torch.isfinite(y[b]).any()
            else:
                check_ffn(y[b:b + 1], own_reference(gate, up, down, group, x[b:b + 1], [sel[b].long()]), 1)


def test_linear_inputs_that_are_not_finite(pb):
    """One input that is not finite, anywhere in a token: all of the token's outputs are NaN, whatever the scales; one block and clusters."""
    for N, K, group in ((272, 512, 128), (40, 14336, 128), (3000, 4096, 32)):
        B = 5
        w = make_w4(N, N, K, group, False, spread=0.01)
        for at in (0, K // 2 + 3, K - 1):
            x = tokens(N, B, K, torch.bfloat16)
            x[1, at], x[3, at] = float("inf"), float("nan")
            x[4] = float("-inf")
            y = torch.empty(B, N, device="cuda")
            pb.prox_w4_linear(w, N, K, group, x, K, 0, B, y, N, 1)
            assert torch.isnan(y[[1, 3, 4]]).all()
            check_linear(y[[0, 2]], w, group, x[[0, 2]], K, 1)
