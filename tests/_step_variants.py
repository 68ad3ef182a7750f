"""Attention calls over the 4-bit cache that between them take every kernel that the dispatch
can choose: how many waves of a workgroup part its keys, into how many workgroups a sequence's
keys are parted, and how the parts are joined.  test_step_plan.py holds the plans to the table
on the CPU, test_gpu_cache4_variants.py runs the calls, each with every type and both head sizes.

Lengths are far below max_tokens where only the plan needs many tokens (a cache's capacity), or
many sequences, so that a case stays small."""

# name: batch, heads, kv_heads, queries, page, max_tokens, lengths of the first sequences (`rest`
# of the others), query counts (None: all), causal, tokens whose pages are missing (sequence,
# token), the plan: waves, parts ("one", "few": joined by one thread each, "many"), and keys of a
# wave that are exceeded (2048 are one look at the page table)
CALLS = {
    "eight": dict(batch=2, heads=14, kv_heads=2, queries=1, page=64, max_tokens=2048,
                  lengths=[2048, 3], plan=dict(waves=8, parts="one")),
    "eight_rows": dict(batch=3, heads=8, kv_heads=2, queries=9, page=32, max_tokens=1500,
                       lengths=[1500, 9, 8], counts=[9, 9, 4], missing=[(0, 700)],
                       plan=dict(waves=8, parts="one")),
    "four_whole": dict(batch=60, heads=16, kv_heads=8, queries=1, page=128, max_tokens=400,
                       lengths=[400, 129, 128, 127, 0], rest=40,
                       plan=dict(waves=4, parts="one")),
    "four_few": dict(batch=10, heads=16, kv_heads=8, queries=3, page=64, max_tokens=2500,
                     lengths=[2500, 513, 512, 511, 2], rest=70, missing=[(0, 0), (0, 1100)],
                     plan=dict(waves=4, parts="few")),
    "four_many": dict(batch=2, heads=14, kv_heads=2, queries=4, page=128, max_tokens=20000,
                      lengths=[9000, 1], plan=dict(waves=4, parts="many")),
    "four_many_all_see_all": dict(batch=2, heads=6, kv_heads=1, queries=9, page=32,
                                  max_tokens=5000, lengths=[4999, 700], causal=False,
                                  counts=[9, 5], missing=[(0, 2000), (1, 0)],
                                  plan=dict(waves=4, parts="many")),
    # a look at the page table more
    "four_long": dict(batch=60, heads=16, kv_heads=8, queries=1, page=64, max_tokens=20000,
                      lengths=[20000, 12801, 2049, 0], rest=33, missing=[(0, 5000), (1, 2100)],
                      plan=dict(waves=4, parts="few", keys=2048)),
    "two_whole": dict(batch=100, heads=8, kv_heads=8, queries=1, page=32, max_tokens=250,
                      lengths=[250, 129, 128, 0], rest=31, plan=dict(waves=2, parts="one")),
    "two_few": dict(batch=100, heads=32, kv_heads=8, queries=2, page=128, max_tokens=6000,
                    lengths=[6000, 2561, 2560, 2, 0], rest=50, missing=[(0, 2600)],
                    plan=dict(waves=2, parts="few")),
    "two_long": dict(batch=120, heads=16, kv_heads=16, queries=1, page=64, max_tokens=9000,
                     lengths=[9000, 8449, 4300], rest=20, missing=[(0, 3000), (2, 4299)],
                     plan=dict(waves=2, parts="few", keys=2048)),
    "one": dict(batch=64, heads=32, kv_heads=32, queries=3, page=64, max_tokens=4400,
                lengths=[4400, 4097, 2050, 2049, 2048, 130, 0], rest=5,
                missing=[(0, 2500), (0, 4399), (1, 4096), (3, 2048)],
                plan=dict(waves=1, parts="one", keys=2048)),
    # many rows, the limits of which lie in the first, the second and the third look
    "one_rows": dict(batch=2, heads=8, kv_heads=4, queries=2100, page=128, max_tokens=4300,
                     lengths=[4300, 2100], counts=[2100, 777], missing=[(0, 3000)],
                     plan=dict(waves=1, parts="one", keys=2048)),
}
DTYPES = ("bf16", "f16", "f32")
HEAD_DIMS = (64, 128)


def lengths_of(c):
    return c["lengths"] + [c.get("rest", 0)] * (c["batch"] - len(c["lengths"]))
