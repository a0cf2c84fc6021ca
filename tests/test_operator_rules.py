"""The rules that cut differential attention and LayerNorm's gradient into workgroups (csrc/jv_plan.h), on the host, and that the GPU
tests reach every variant they choose among."""
import shutil

import pytest

import test_gpu_diff_attn_variants as V
import test_gpu_layernorm_bwd
from test_dispatch_rules import rule  # noqa: F401  (a fixture)

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def plan(rule, cases):  # noqa: F811
    """[(waves, blocks, splits, tiles_per_split)] of (B, kv_heads, rows, n_k, W, bf16)"""
    call = [f"diff_plan({B}, {G}, {rows}ll, {n_k}, {W}, {int(bf16)})" for B, G, rows, n_k, W, bf16 in cases]
    got = rule([f"{c}.{f}" for c in call for f in ("waves", "blocks", "splits", "tiles_per_split")])
    return [tuple(got[i:i + 4]) for i in range(0, len(got), 4)]


def test_plans_of_the_forward_pass(rule):  # noqa: F811
    cases = [(B, G, rows, n_k, W, bf16) for B, G in ((1, 1), (2, 8), (65535, 1), (1, 65535)) for rows in (1, 16, 17, 32, 64, 65, 128, 129, 1 << 24, 1 << 30)
             for n_k in (1, 32, 33, 64, 255, 256, 1000, 1 << 14, 1 << 24) for W in (64, 128) for bf16 in (False, True)]
    for (B, G, rows, n_k, W, bf16), (waves, blocks, splits, per) in zip(cases, plan(rule, cases)):
        tiles, groups = (n_k + 31) // 32, B * G * blocks
        assert waves == (1 if rows <= 64 else 4) and 32 * waves * (blocks - 1) < rows <= 32 * waves * blocks
        # no part without a tile, none missing, and no more than a launch or the join takes
        assert 1 <= splits <= 256 and per * splits >= tiles and per * (splits - 1) < tiles
        holds = 768 if waves == 1 and (bf16 or W == 128) else 1536 if waves == 1 else 512 if bf16 or W == 64 else 256
        alone = not bf16 and W == 128 and waves > 1 and groups > 16   # see test_parts_of_workgroups_with_a_unit_each
        assert splits == 1 or (splits <= 16 if alone else groups * splits <= holds)
        assert not bf16 or splits == 1 or per >= (2 if rows <= 16 else 4)


def test_the_gpu_tests_reach_every_join(rule):  # noqa: F811
    def kind(splits):
        return 1 if splits == 1 else 2 if splits == 2 else 4 if splits <= 4 else 8 if splits <= 8 else 9 if splits <= 32 else 33 if splits <= 64 else 65
    for bf16 in (False, True):
        for W in (64, 128):
            cases = [(1, 1, h * n, n_k, W, bf16) for h, n in V.ROWS for n_k in V.KEYS]
            kinds = {}
            for c, (waves, _, splits, _) in zip(cases, plan(rule, cases)):
                kinds.setdefault((waves, bf16 and c[2] <= 16), set()).add(kind(splits))
            assert set(kinds) == ({(1, True), (1, False), (4, False)} if bf16 else {(1, False), (4, False)})
            assert all(k == {1, 2, 4, 8, 9, 33, 65} for k in kinds.values()), (bf16, W, kinds)


def test_parts_of_the_gradient(rule):  # noqa: F811
    cases = [(items, tiles, b, c) for items in (1, 3, 31, 32, 33, 256, 257, 512, 513, 1024, 1025, 65535 << 17) for tiles in (1, 3, 4, 5, 8, 64, 1000, 1 << 19)
             for b in (0, 1) for c in (0, 1)]
    got = rule([f"diff_bwd_parts({i}ll, {t}ll, {b}, {c})" for i, t, b, c in cases])
    for (items, tiles, bf16, causal), parts in zip(cases, got):
        assert 1 <= parts <= 16 and parts <= max(1, tiles // (4 if bf16 else 2))
        if bf16 or causal:
            assert parts == 1 or items * parts <= (512 if bf16 else 256) * (2 if causal else 1)
    for bf16 in (0, 1):   # what the GPU tests reach: one part, several, and the most, of either pass
        q, k = set(), set()
        for B, H, G, n_q, n_k, causal in V.GRADIENTS:
            blocks, tiles = [(n + 127) // 128 for n in (n_q, n_k)], [(n + 31) // 32 for n in (n_q, n_k)]
            p = rule([f"diff_bwd_parts({B * H * blocks[0]}, {tiles[1]}, {bf16}, {int(causal)})",
                      f"diff_bwd_parts({B * G * blocks[1]}, {tiles[0] * (H // G)}, {bf16}, {int(causal)})"])
            q.add(p[0])
            k.add(p[1])
        for parts in (q, k):
            assert 1 in parts and 16 in parts and parts & set(range(2, 16)), (bf16, q, k)


def test_parts_of_workgroups_with_a_unit_each(rule):  # noqa: F811
    """No number of parts up to 16 of two tiles takes fewer tiles one after the other, by the rule's count of them."""
    cases = [(items, tiles) for items in (1, 17, 100, 128, 129, 132, 256, 257, 288, 511, 5000, 1 << 30) for tiles in (1, 2, 3, 8, 18, 43, 94, 1 << 19)]
    for (items, tiles), got in zip(cases, rule([f"diff_parts_alone({i}ll, {t}ll)" for i, t in cases])):
        time = {p: -(-items * p // 256) * (-(-tiles // p) + (4 if p > 1 else 2)) + (3 if p > 1 else 0) for p in range(1, 17) if p == 1 or 2 * p <= tiles}
        assert time[got] == min(time.values()) and got == min(p for p in time if time[p] == time[got])


def test_rows_and_workgroups_of_a_norm(rule):  # noqa: F811
    cols = [8 * i for i in range(1, 1025)]
    lanes, pieces = rule([f"norm_grad_lanes({c})" for c in cols]), rule([f"norm_grad_pieces({c})" for c in cols])
    for c, n, p in zip(cols, lanes, pieces):
        assert (n, p) in {(8, 1), (16, 1), (32, 1), (64, 1), (64, 2), (128, 2), (256, 2), (512, 2)}
        assert c <= 8 * n * p and (n == 8 or c > 4 * n * p), c   # at most half of the lanes' columns lie behind the row
    sizes = [(r, c) for r in (1, 63, 64, 16384, 16385, 32768, 32769, 65536, 65537, 1 << 31) for c in (8, 64, 128, 1024, 8192)]
    for (r, c), g in zip(sizes, rule([f"norm_grad_groups({r}ll, {c})" for r, c in sizes])):
        per = 512 // lanes[c // 8 - 1]
        steps = (r + per - 1) // per
        assert 1 <= g <= min(steps, 512)
    reached = test_gpu_layernorm_bwd.SIZES + V.NORMS
    assert {lanes[c // 8 - 1] * pieces[c // 8 - 1] for _, c in reached} == {8, 16, 32, 64, 128, 256, 512, 1024}
    per_group = set()
    for (r, c), g in zip(reached, rule([f"norm_grad_groups({r}, {c})" for r, c in reached])):
        steps = -(-r // (512 // lanes[c // 8 - 1]))
        per_group.add("one" if g == steps else "two" if g == (steps + 1) // 2 else "256" if g == 256 else "512")
    assert per_group == {"one", "two", "256", "512"}
