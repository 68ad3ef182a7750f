"""Attention calls that between them take every kernel that the dispatch can choose: the call
and what e2s_cache_attend's plan has to say of it.  test_serve_plan.py holds the plans to the
table on the CPU, test_gpu_cache_variants.py runs the calls.

Lengths are far below max_tokens where only the plan needs many tokens (a cache's capacity),
so that a case stays small."""

# name: dtype, batch, heads, kv_heads, queries, head_dim, page, max_tokens, lengths of the first
# sequences (`rest` of the others), query counts (None: all), causal, weights, the plan
CALLS = {
    # a prompt: 32 rows to a wave, more than 64 steps (a second look at the page table), rows
    # that see nothing, fewer queries than there is room for
    "prompt_bf16_128": dict(
        dtype="bf16", batch=4, heads=8, kv_heads=8, queries=2048, head_dim=128, page=64,
        max_tokens=4300, lengths=[4300, 3001, 700, 0], counts=[2048, 1000, 2048, 3], weights=True,
        plan=dict(shared_rows=1, tiles=2, waves=4, splits=1, lse_kept=1, steps=64)),
    "prompt_bf16_64_all_see_all": dict(
        dtype="bf16", batch=8, heads=64, kv_heads=64, queries=65, head_dim=64, page=16,
        max_tokens=300, lengths=[300, 299, 65, 64], rest=17, causal=False,
        plan=dict(shared_rows=1, tiles=2, waves=4, splits=1)),
    # queries in two and three parts keep 16 rows to a wave; more than 64 steps again
    "prompt_f16_128": dict(
        dtype="f16", batch=16, heads=8, kv_heads=8, queries=300, head_dim=128, page=128,
        max_tokens=16384, lengths=[5300, 301, 300, 12], rest=20, weights=True,
        counts=[300, 300, 299, 300] + [1] * 12,
        plan=dict(shared_rows=1, tiles=1, waves=4, steps=64, few_parts=1)),
    "prompt_f32_64": dict(
        dtype="f32", batch=2, heads=4, kv_heads=2, queries=150, head_dim=64, page=32,
        max_tokens=1500, lengths=[1500, 77], weights=True,
        plan=dict(shared_rows=1, tiles=1, waves=4, few_parts=1)),
    "run_bf16_128_many_parts": dict(
        dtype="bf16", batch=2, heads=8, kv_heads=2, queries=12, head_dim=128, page=64,
        max_tokens=20000, lengths=[9000, 3], weights=True,
        plan=dict(shared_rows=1, tiles=1, waves=4, few_parts=0)),
    # 17 to 32 rows whose waves part the keys
    "two_tiles_parts_bf16_128": dict(
        dtype="bf16", batch=2, heads=14, kv_heads=2, queries=4, head_dim=128, page=64,
        max_tokens=2500, lengths=[2500, 1], weights=True,
        plan=dict(shared_rows=0, tiles=2, waves=4, few_parts=0)),
    "two_tiles_parts_f16_64": dict(
        dtype="f16", batch=2, heads=14, kv_heads=2, queries=4, head_dim=64, page=16,
        max_tokens=2500, lengths=[2499, 3], counts=[4, 2], weights=True,
        plan=dict(shared_rows=0, tiles=2, waves=4, few_parts=0)),
    "two_tiles_parts_f32_128": dict(
        dtype="f32", batch=1, heads=6, kv_heads=2, queries=10, head_dim=128, page=32,
        max_tokens=2200, lengths=[2050], weights=True,
        plan=dict(shared_rows=0, tiles=2, waves=4)),
    # one query of many or long sequences at d = 128
    "one_bf16_128_many_parts": dict(
        dtype="bf16", batch=3, heads=8, kv_heads=2, queries=1, head_dim=128, page=64,
        max_tokens=20000, lengths=[6001, 50, 0], weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=4, few_parts=0)),
    "one_f32_128_many_parts": dict(
        dtype="f32", batch=2, heads=8, kv_heads=2, queries=1, head_dim=128, page=32,
        max_tokens=9000, lengths=[9000, 255], weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=4, few_parts=0)),
    "one_f16_128_few_parts": dict(
        dtype="f16", batch=20, heads=32, kv_heads=8, queries=1, head_dim=128, page=16,
        max_tokens=6000, lengths=[6000, 2047, 2049], rest=9, weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=4, few_parts=1)),
    # a workgroup's waves have more than 64 tiles each: a second look at the page table
    "one_bf16_128_long_parts": dict(
        dtype="bf16", batch=75, heads=8, kv_heads=4, queries=1, head_dim=128, page=128,
        max_tokens=32768, lengths=[32768, 9000, 4864, 4865], rest=7,
        plan=dict(shared_rows=0, tiles=1, waves=4, few_parts=1, quarter=1024)),
    # full devices: nothing is split, and the weights are a launch of their own
    "one_f16_64_full": dict(
        dtype="f16", batch=32, heads=64, kv_heads=64, queries=1, head_dim=64, page=32,
        max_tokens=5000, lengths=[5000, 1281, 0], rest=33, weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=4, splits=1, lse_kept=1, quarter=1024)),
    "one_bf16_128_full": dict(
        dtype="bf16", batch=128, heads=32, kv_heads=8, queries=1, head_dim=128, page=64,
        max_tokens=1000, lengths=[1000, 0, 1], rest=100, weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=4, splits=1, lse_kept=1)),
    "two_tiles_f32_64_full": dict(
        dtype="f32", batch=128, heads=24, kv_heads=8, queries=6, head_dim=64, page=16,
        max_tokens=128, lengths=[128, 5, 0], rest=60, counts=[6, 6, 6] + [2] * 125, weights=True,
        plan=dict(shared_rows=0, tiles=2, waves=4, splits=1, lse_kept=1)),
    # short sequences: eight waves
    "eight_waves_bf16_128": dict(
        dtype="bf16", batch=40, heads=32, kv_heads=8, queries=1, head_dim=128, page=64,
        max_tokens=2000, lengths=[2000, 256, 0, 1], rest=90, weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=8, splits=1, lse_kept=0)),
    "eight_waves_one_sequence": dict(
        dtype="bf16", batch=1, heads=8, kv_heads=2, queries=1, head_dim=128, page=64,
        max_tokens=1024, lengths=[1024], weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=8, splits=1)),
    "parts_of_one_sequence": dict(
        dtype="bf16", batch=1, heads=8, kv_heads=2, queries=1, head_dim=128, page=64,
        max_tokens=1025, lengths=[1025], weights=True,
        plan=dict(shared_rows=0, tiles=1, waves=4, few_parts=1)),
    "eight_waves_two_tiles_bf16_128": dict(
        dtype="bf16", batch=2, heads=14, kv_heads=2, queries=4, head_dim=128, page=32,
        max_tokens=700, lengths=[700, 3], weights=True,
        plan=dict(shared_rows=0, tiles=2, waves=8, splits=1, lse_kept=0)),
}


def lengths_of(c):
    return c["lengths"] + [c.get("rest", 0)] * (c["batch"] - len(c["lengths"]))
