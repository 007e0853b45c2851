"""The rules of csrc/jet_step_plan.h: every kernel is met by a case of test_gpu_step.py, and what the kernels take for granted holds."""
import step_plan as plan
import test_gpu_step as gpu
import test_gpu_step_calls as calls


def test_the_cases_meet_every_way_to_order_tokens():
    n, L = plan.numbers(), plan.lib()
    assert n["places"] <= n["sort_block"] and n["direct"] % 64 == 0 and n["narrow_rows"] * n["sort_block"] < 1 << 32
    assert {plan.order(c[0]) for c in gpu.EMBED} == {"direct", "places", "sort"}
    assert {c[0] for c in gpu.EMBED} >= {n["direct"], n["direct"] + 1, n["places"], n["places"] + 1}
    sizes = {L.block(c[0], c[1]) for c in gpu.EMBED if plan.order(c[0]) != "direct"}
    assert sizes == {8, 16, 32}
    assert any(c[2] > n["narrow_rows"] and plan.order(c[0]) == "sort" for c in gpu.EMBED)
    # runs that are merged: none, once and twice, with a last run of its own; the one whose length is a power of two
    rank, each, runs = n["rank_tokens"], n["rank_blocks"] * n["sort_block"], n["merge_runs"]
    assert each & (each - 1) == 0 and runs & (runs - 1) == 0 and each <= rank
    assert [L.merges(T) for T in (1, rank, rank + 1, each * runs, each * runs + 1, 1 << 22)] == [0, 0, 1, 1, 2, 2]
    assert {L.merges(c[0]) for c in gpu.EMBED} == {L.merges(T) for T in gpu.ONE_ROW} == {0, 1, 2}
    # few tokens, whose sums are those of a row or of so many tokens
    places = [c for c in gpu.EMBED if plan.order(c[0]) == "places"]
    assert {L.by_runs(c[0], c[1]) for c in places} == {0, 1} and {c[0] for c in places if L.by_runs(c[0], c[1])} >= {n["direct"] + 1, n["places"]}
    # zeros of the second launch: none, some, as many as it takes
    sizes = [c[2] * c[1] * b for c in gpu.EMBED for b in (2, 4) if plan.order(c[0]) == "sort"]
    most = L.later(1 << 40)
    assert all(0 <= L.later(b) <= min(b, most) and L.later(b) % 16 == 0 for b in sizes)
    assert {min(1, L.later(b)) + (L.later(b) == most) for b in sizes} == {0, 1, 2}
    # a row of more and one of fewer blocks than those that are joined by themselves
    for T in gpu.ONE_ROW:
        if plan.order(T) != "direct":
            assert T > (n["long_run"] + 2) * L.block(T, 1032)


def test_embedding_workspace():
    L, n = plan.lib(), plan.numbers()
    for T in (1, 256, 257, 1000, 1024, 1025, 2049, 40000, 1 << 22):
        for H in (8, 1000, 4096):
            tmp, partial, size = (L.space(T, H, i) for i in range(3))
            if plan.order(T) == "direct":
                assert size == 0
                continue
            padded = -(-T // n["sort_block"]) * n["sort_block"] * 4
            assert tmp == 2 * padded and partial == (2 * tmp if plan.order(T) == "sort" else tmp)
            b = L.block(T, H)
            assert b in (8, 16, 32) and size == partial + (0 if L.by_runs(T, H) else -(-T // b) * 2 * H * 4)
            assert plan.order(T) == "places" or not L.by_runs(T, H)
            assert size % 16 == 0 and partial % 16 == 0


def test_the_cases_meet_every_team_of_a_row():
    for K in list(range(8, 32769, 8)):
        for waves, pieces in [plan.bwd_team(K)] + [plan.team(M, K, both) for M in (1, 1024, 1025) for both in (False, True)]:
            assert waves * pieces * 512 >= K and 1 <= waves <= 16 and pieces in (1, 2, 4)
            assert waves > 1 or pieces < 4
    kind = lambda t: (t[0] > 1, t[1])
    assert {kind(plan.team(M, K)) for M, K in gpu.NORMS} == {(False, 1), (False, 2), (True, 1), (True, 2), (True, 4)}
    assert {kind(plan.bwd_team(K)) for _, K in gpu.NORMS} == {(False, 1), (False, 2), (True, 1), (True, 2), (True, 4)}
    assert {plan.team(M, K) for M, K in gpu.NORMS if 512 < K <= 1024} == {(1, 2), (2, 1)}
    both = {K: {plan.team(M, K) for M in (1, gpu.MANY)} for K in gpu.SAME_BYTES}
    assert all(len(t) == 2 for K, t in both.items() if 512 < K <= 8192) and len(both) > 5
    # rows that a team takes one after the other: none, fewer than are under way, many
    rows = {-(-M // (plan.lib().bwd_groups(M, K) * (4 if plan.bwd_team(K)[0] == 1 else 1))) for M, K in gpu.NORMS}
    assert {1, 2, 3, 4} <= rows and max(rows) > 8


def test_the_cases_meet_both_sides_of_every_size():
    n, L = plan.numbers(), plan.lib()
    for shape in gpu.PAST_THE_CACHES:
        assert L.nt(2 * shape[0] * shape[1])
    # threads of layer norm's largest launches: 64 for each 512 columns
    for K in range(8, 32769, 8):
        M = min(1 << 23, (1 << 34) // K)
        assert all(M * 64 * plan.team(M, K, both)[0] < 1 << 32 for both in (False, True))
    assert not any(L.nt(2 * M * K) for M, K in gpu.NORMS) and not all(L.nt(2 * c[0] * c[1]) for c in gpu.EMBED)
    size = lambda t: sum((v if isinstance(v, int) else v[0] * v[1]) * (2 if i % 3 else 4) for i, v in enumerate(t))
    assert any(size(t) > max(n["fuse"], n["keep"]) and len(t) <= n["batch"] for t in gpu.CLIP)
    assert any(size(t) > max(n["fuse"], n["keep"]) and len(t) > n["batch"] for t in gpu.CLIP)
    assert any(size(t) < n["fuse"] and len(t) > n["batch"] for t in gpu.CLIP)
    assert any(n["groups"] * n["chunk"] < sum(v if isinstance(v, int) else v[0] * v[1] for v in t) for t in gpu.CLIP)


def test_the_norm_is_not_added_up_again_by_every_workgroup():
    """Work of the second pass on partial sums: as many as one launch makes, in each workgroup, or none."""
    n, L = plan.numbers(), plan.lib()

    def sums(sizes):
        chunks = [-(-v // n["chunk"]) for v in sizes if v]
        return sum(L.clip_sums(sum(chunks[i:i + n["batch"]])) for i in range(0, len(chunks), n["batch"]))

    assert L.norm_alone(n["fuse"] + 1, 1) and not L.norm_alone(n["fuse"], n["groups"]) and L.norm_alone(1000, n["groups"] + 1)
    assert sums([1000] * 65536) == 65536 and L.norm_alone(65536 * 2000, 65536)
    # the cases of test_gpu_step_calls.py: many tensors, many bytes, neither
    size = lambda sizes: sum(v * (2 if i % 3 else 4) for i, v in enumerate(sizes))
    assert all(sums(t) > n["groups"] and size(t) <= n["fuse"] for t in calls.MANY_TENSORS)
    assert sums(calls.LARGE) <= n["groups"] and size(calls.LARGE) > n["fuse"]
    assert sums(calls.FEW) <= n["groups"] and size(calls.FEW) <= n["fuse"]


def test_workgroups_of_the_norm_gradients_run_at_once():
    """Each keeps sums that the second launch reads, so none waits for another: as many waves as 256 CUs hold, 16 each where a lane has more than one piece
    (up to 128 registers), else 20 (up to 96)."""
    L = plan.lib()
    for K in range(8, 32769, 8):
        waves, pieces = plan.bwd_team(K)
        for M in (1, 500, 1100, 4096, 1 << 19):
            groups = L.bwd_groups(M, K)
            assert 1 <= groups <= 512 and groups * max(waves, 4) <= 256 * (16 if pieces > 1 else 20), (M, K)
