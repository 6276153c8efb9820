"""prox_token_logprobs: one logit that is no number, or +inf, makes every log probability and the entropy of its row NaN, wherever
in the row it lies.  A block takes a row, or its share of one, in rounds of 16384 16-bit or 8192 32-bit logits; places are
taken from the first, a middle and the last round, from the ends of the row, and (few rows) from every block of a cluster."""
import pytest
import torch

from tests.test_gpu_logprobs import DT, call, check, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pb():
    import __graft_entry__ as entry
    entry.build()
    from paper_2607_27591_b200 import binding
    return binding


def places(V, per_round):
    """A place in every round, two in the first and last, both ends, and sixteen spread over the row."""
    at = {0, 1, V - 1, V - 2, V // 2, min(V - 1, 777)}
    at |= {min(V - 1, r + 4099) for r in range(0, V, per_round)} | {V * i // 16 + 3 for i in range(16)}
    return sorted(at)


def rows_with_one(value, T, V, dt, seed):
    x = (torch.randn(T, V, device="cuda", generator=gen(seed)) * 2).to(DT[dt])
    spots = places(V, 8192 if dt == 1 else 16384)
    bad = {}
    for i, at in enumerate(spots):                              # every other row stays whole
        if 2 * i + 1 < T:
            bad[2 * i + 1] = at
            x[2 * i + 1, at] = value
    return x, bad


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("V", [20000, 131072, 100003])
@pytest.mark.parametrize("dt", [0, 1, 2])
def test_one_logit_in_any_round(pb, dt, V, top, value):
    """A block per row."""
    T = 160
    x, bad = rows_with_one(value, T, V, dt, V + dt)
    ids = torch.randint(0, V, (T, 3), device="cuda", generator=gen(1), dtype=torch.int32)
    lp, en, tl, ti = call(pb, x, dt, V, 1.0, ids, top)
    whole = [r for r in range(T) if r not in bad]
    check(x[whole], V, 1.0, ids[whole], top, (lp[whole], en[whole], tl[whole], ti[whole]))
    spoilt = sorted(bad)
    assert torch.isnan(lp[spoilt]).all() and torch.isnan(en[spoilt]).all() and torch.isnan(tl[spoilt]).all()
    if top:
        assert ti[spoilt, 0].tolist() == [bad[r] for r in spoilt]


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("top", [0, 6])
@pytest.mark.parametrize("dt", [0, 1, 2])
def test_one_logit_in_any_block_of_a_cluster(pb, dt, top, value):
    """Few rows: every row is split over blocks, which still have several rounds each."""
    T, V = 2, 600001
    for at in [0, 5, V - 1] + [V * i // 16 + 11 for i in range(16)]:
        x = (torch.randn(T, V, device="cuda", generator=gen(at)) * 2).to(DT[dt])
        x[1, at] = value
        ids = torch.randint(0, V, (T, 2), device="cuda", generator=gen(2), dtype=torch.int32)
        lp, en, tl, ti = call(pb, x, dt, V, 1.0, ids, top)
        check(x[:1], V, 1.0, ids[:1], top, (lp[:1], en[:1], tl[:1], ti[:1]))
        assert torch.isnan(lp[1]).all() and torch.isnan(en[1]) and torch.isnan(tl[1]).all()
        if top:
            assert int(ti[1, 0]) == at


@pytest.mark.parametrize("dt", [0, 1, 2])
def test_a_thread_keeps_what_it_has_seen(pb, dt):
    """Rows whose later rounds hold nothing but -inf, or nothing above the first: with a NaN early on, and without one."""
    T, V = 200, 70001
    x = torch.full((T, V), float("-inf"), device="cuda", dtype=DT[dt])
    x[:, :1000] = (torch.randn(T, 1000, device="cuda", generator=gen(5)) + 8).to(DT[dt])
    x[100:, 1000:] = (torch.randn(100, V - 1000, device="cuda", generator=gen(6)) - 8).to(DT[dt])
    x[1::2, 17] = float("nan")
    ids = torch.randint(0, V, (T, 2), device="cuda", generator=gen(7), dtype=torch.int32)
    lp, en, tl, ti = call(pb, x, dt, V, 1.0, ids, 4)
    check(x[0::2], V, 1.0, ids[0::2], 4, (lp[0::2], en[0::2], tl[0::2], ti[0::2]))
    assert torch.isnan(lp[1::2]).all() and torch.isnan(en[1::2]).all() and torch.isnan(tl[1::2]).all()
