"""The cases that the GPU tests take reach every instance that the decoder's calls choose from (no GPU)."""
import itertools

import decoder_cases as cases
import decoder_reference as ref
import pytest
import torch

BOTH = (64, 128)


def _dims(case):
    return BOTH if case[0] == 0 else case[:1]


def test_attention_over_the_cache():
    reached = set()
    for case, want in cases.ATTEND:
        for d in _dims(case):
            assert cases.attend_plan(d, *case[1:]) == want, (d, case)
            reached.add((d, *want))
    # one tile of 16 rows and two, four waves and eight: alone and shared, with the least shares and not; many rows: eight
    want = {(d, t, w, s, f) for d, (t, w), (s, f) in itertools.product(BOTH, [(1, 4), (1, 8), (2, 4), (2, 8), (8, 8)], [(0, 0), (1, 0), (1, 1)])}
    assert reached == want | {(64, 1, 16, 0, 0)}


@pytest.mark.parametrize("d, keys, most", [(64, 1024, 192), (64, 4096, 192), (64, 4097, 128), (64, 30000, 128), (128, 1024, 64), (128, 9000, 64)])
def test_rows_of_a_tile(d, keys, most):
    """The borders where tiles of 128 rows are the faster ones, as measured (128 rows to 192 at d = 64 are not, with few keys)."""
    for G in (1, 4):
        tiles = [cases.internal_plan("cached", 8, 12 * G, 12, rows // G, keys, d)[0] for rows in (4, 16, 20, most, most + 4, 2048)]
        assert tiles == [1, 1, 2, 2, 8, 8]


@pytest.mark.parametrize("d", BOTH)
def test_shares_of_few_blocks_have_eight_waves(d):
    """As measured: sequences that are few for the chip are walked by eight waves to a workgroup, however few blocks they have in all."""
    for B, Hk, queries, keys in ((1, 8, 1, 6000), (1, 2, 1, 32768), (4, 8, 1, 8192), (2, 8, 8, 8192)):
        assert cases.internal_plan("cached", B, 4 * Hk, Hk, queries, keys, d)[1:3] == (8, 1)


def test_who_walks_five_blocks_and_who_fewer():
    """As measured: few workgroups of long blocks share their keys from 33 blocks on, of 128 rows from 25, others from 41."""
    for d, B, Hk, queries, most in ((64, 1, 8, 1, 80), (64, 1, 8, 8, 40), (128, 1, 8, 1, 32), (128, 8, 8, 1, 32), (128, 12, 8, 1, 40), (128, 8, 8, 8, 32), (64, 1, 8, 256, 24), (64, 2, 8, 256, 40),
                                    (128, 1, 8, 256, 24), (128, 2, 8, 256, 40)):
        shared = [cases.internal_plan("cached", B, 4 * Hk, Hk, queries, keys, d)[2] for keys in (64 * most, 64 * most + 1)]
        assert shared == [0, 1], (d, B, Hk, queries)


def test_append():
    reached = set()
    for case, want in cases.APPEND:
        assert cases.append_plan(*case) == want, case
        reached.add((case[0], *want, case[-1] == "prompt"))
    units = {64: [(1, 1), (1, 2), (1, 4), (4, 2), (4, 4)], 128: [(1, 1), (1, 2), (1, 4), (4, 2), (4, 4), (4, 8)]}
    assert {x[:4] for x in reached} == {(d, *u, each) for d in BOTH for u in units[d] for each in (1, 2, 4)}
    assert {x[3] for x in reached if x[4]} == {1, 2, 4}
    # (nothing else is ever chosen)
    for d, page, Hk, B, new in itertools.product(BOTH, (16, 32, 64, 128), (1, 16), (1, 70), (1, 2, 5, 9, 17, 40, 100, 400)):
        for ragged in (0, 1):
            waves, passes, _ = cases.internal_plan("append", B * new, ragged, B, new, page, Hk, d)
            assert passes <= (4 if waves == 1 else 8 * units[d][-1][1] // 2) and (waves == 1) == (passes <= 4)


def test_norm():
    reached = set()
    for case, want in cases.NORM:
        assert cases.norm_plan(*case) == want, case
        reached.add((case[0], case[1], *want))
    forward, backward = {x[:4] for x in reached}, {(*x[:2], x[4]) for x in reached}
    assert forward == {(t, d, u, p) for t, d, u, p in itertools.product(("bf16", "f32"), BOTH, (1, 4), (0, 1)) if not (t == "f32" and p)}
    assert backward == set(itertools.product(("bf16", "f32"), BOTH, (0, 1)))


@pytest.mark.parametrize("mode", [(2, 4), (1, 2), (0, 0)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_a_sequence_at_once_is_its_queries_one_by_one(causal, mode):
    g = torch.Generator().manual_seed(70)
    lengths, counts = [37, 5, 0, 64], [6, 7, 2, 1]
    Q = torch.randn(sum(counts), 4, 8, generator=g, dtype=torch.float64)
    K, V = ([torch.randn(2, n, 8, generator=g, dtype=torch.float64) for n in lengths] for _ in range(2))
    seen = [torch.rand(n, generator=g) > 0.2 for n in lengths]
    for a, b in zip(ref.attention(Q, counts, K, V, seen, lengths, 50, *mode, 0.3, causal), ref.attention_at_once(Q, counts, K, V, seen, lengths, 50, *mode, 0.3, causal)):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)


def test_appended_heads_at_once_are_one_by_one():
    g = torch.Generator().manual_seed(71)
    table, lengths, counts = torch.tensor([[3, 0, 9], [1, 4, 2]], dtype=torch.int32), [20, 47], [18, 20]
    x = torch.randn(38, 3, 64, generator=g, dtype=torch.float64) * 300
    values, scale = ref.nearest(torch.randn(6, 3, 16, 64, generator=g, dtype=torch.float64)), torch.full((6, 3), 0.25, dtype=torch.float64)
    one, at_once = [(values.clone(), scale.clone()) for _ in range(2)]
    args = (x, table, lengths, counts, 16, 45, 6)
    assert torch.equal(ref.append(*one, *args).nan_to_num(nan=7.0), ref.append_at_once(*at_once, *args).nan_to_num(nan=7.0))
    assert all(torch.equal(a, b) for a, b in zip(one, at_once)) and not torch.equal(one[0], values)
