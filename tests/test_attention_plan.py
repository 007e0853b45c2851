"""The rules that pick the attention operators' kernels (csrc/jet_attn_plan.h), on the host: a changed rule would take a kernel out of the
GPU tests without any of them failing."""
import pytest

import attention_plan as plan
from test_gpu_attention import DECODE, PACKED
from test_gpu_attention_large import FEW, LARGE
from test_gpu_attention_qk import MANY, MANY_BWD, MANY_KEPT


@pytest.mark.parametrize("case", LARGE, ids=lambda c: f"{len(c[0])}x{max(c[0])}+{c[1]}-{c[2]}.{c[3]}.{c[4]}-{c[5]}")
def test_the_large_cases_run_the_kernels_of_many_tiles(case):
    assert plan.rows(case) == "many" and plan.keys(case)[0] == "many"
    assert max(case[0]) + case[1] > 2 * 256                   # past the keys for which delta has a pass of its own, and many blocks


def test_the_large_cases_cover_widths_masks_and_pieces():
    seen = {(c[4], c[5]) for c in LARGE}
    assert seen == {(64, False), (64, True), (128, False), (128, True)}
    for dim, causal in seen:
        pieces = [p for c in LARGE if c[4:] == (dim, causal) for p in plan.keys(c)[1]]
        assert max(pieces) >= 2, (dim, causal)                # joined sums
        assert dim == 64 or 1 in pieces or not causal
    assert any(1 in plan.keys(c)[1] and max(plan.keys(c)[1]) > 1 for c in LARGE)        # both in one call
    assert any(max(plan.keys(c)[1]) == 8 for c in LARGE)
    groups = [c[2] // c[3] for c in LARGE]
    assert any(32 % g for g in groups) and any(g == 1 for g in groups) and any(g > 16 for g in groups)
    assert any(c[1] for c in LARGE) and any(0 in c[0] for c in LARGE)
    ends = {(n + c[1]) % 64 for c in LARGE for n in c[0]}
    assert {0, 1} <= ends and len(ends) > 10


@pytest.mark.parametrize("case", FEW)
def test_the_few_cases_run_the_kernels_of_few_tiles_over_many_keys(case):
    assert plan.rows(case) == "few" and plan.keys(case)[0] == "few" and max(case[0]) + case[1] > 256


def test_the_packed_cases_run_the_kernels_of_few_tiles():
    def sizes(c):
        lk = c[0] if c[1] is None else c[1]
        return len(c[0]), sum(c[0]), sum(lk), c[2] // c[3], c[3], c[4]
    few = [c for c in PACKED if plan.lib().few_rows(*sizes(c))]
    assert {(c[4], c[5]) for c in few} == {(64, False), (64, True), (128, False), (128, True)}


def test_decode_cases_have_one_chunk_and_several():
    seen = set()
    for lengths, n_q, n_kv, dim, page, spare in DECODE:
        width = max(1, -(-max(lengths) // page)) + spare
        for fp8 in (False, True):
            seen.add((dim, fp8, min(2, plan.chunks(len(lengths), n_q, n_kv, dim, fp8, width * page))))
    assert seen == {(d, f, n) for d in (64, 128) for f in (False, True) for n in (1, 2)}


def test_the_cases_of_many_tokens_run_four_heads_to_a_team():
    assert all(plan.heads(*c[:4]) == 4 for c in MANY)
    assert all(plan.heads_bwd(*c[:4]) == 4 for c in MANY_BWD)
    assert all(plan.heads(*c[:4], True) == 4 for c in MANY_KEPT)
    for cases in (MANY, MANY_BWD):
        assert {c[3:] for c in cases} == {(64, True), (64, False), (128, True), (128, False)}
        assert any(c[1] % 4 for c in cases) and any(c[2] % 4 for c in cases)
    assert {(c[3], c[5]) for c in MANY_KEPT} == {(64, False), (64, True), (128, False), (128, True)}
