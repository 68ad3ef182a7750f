"""How an attention call over the 4-bit cache is cut (step_validate.cpp's attend4_plan), without
a GPU: the calls of _step_variants.py take the kernels that they are there for; and the
reference that they are compared with is the plain one."""
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import _step_helpers as H
import _step_variants as V

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_23253_amd", "csrc")
CODES = {"f32": 0, "bf16": 1, "f16": 2}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """The plan of every call, type and head size."""
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = tmp_path_factory.mktemp("plan") / "step_plan"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
           os.path.join(ROOT, "tests", "native", "step_plan.cpp"),
           *(os.path.join(CSRC, n) for n in ("step_validate.cpp", "serve_validate.cpp",
                                             "e2s_validate.cpp")), "-o", str(exe)]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    keys = [(n, kind, d) for n in V.CALLS for kind in V.DTYPES for d in V.HEAD_DIMS]
    lines = []
    for n, kind, d in keys:
        c = V.CALLS[n]
        lines.append(" ".join(str(x) for x in (
            c["page"], c["kv_heads"], d, c["batch"], c["heads"], c["queries"], CODES[kind],
            c["max_tokens"], int(c.get("causal", True)))))
    run = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True,
                         timeout=300)
    assert run.returncode == 0, run.stderr
    names = ("status", "waves", "chunk", "splits", "bytes")
    said = [dict(zip(names, map(int, x.split()[1:]))) for x in run.stdout.splitlines()]
    return dict(zip(keys, said))


@pytest.mark.parametrize("name", V.CALLS)
def test_calls_take_their_kernels(plans, name):
    c = V.CALLS[name]
    want = c["plan"]
    for kind in V.DTYPES:
        for d in V.HEAD_DIMS:
            p = plans[name, kind, d]
            assert p["status"] == 0 and p["waves"] == want["waves"], p
            parts = p["splits"]
            assert want["parts"] == ("one" if parts == 1 else "few" if parts <= 8 else "many"), p
            assert (parts > 1) == (p["bytes"] > 0), p
            # the longest sequence's first workgroup has more keys to a wave
            longest = min(max(V.lengths_of(c)), p["chunk"])
            assert longest / p["waves"] > want.get("keys", 0), p
            if parts > 1:
                assert max(V.lengths_of(c)) > p["chunk"], "a second part with keys"


def test_every_kernel_is_taken():
    taken = {(c["plan"]["waves"], c["plan"]["parts"]) for c in V.CALLS.values()}
    assert taken >= {(8, "one"), (4, "one"), (4, "few"), (4, "many"), (2, "one"), (2, "few"),
                     (1, "one")}
    for waves in (4, 2, 1):
        assert any(c["plan"]["waves"] == waves and "keys" in c["plan"] for c in V.CALLS.values())


@pytest.mark.parametrize("d,P,kind,causal", [(64, 32, "f32", True), (128, 64, "bf16", False)])
def test_the_reference_by_rows_is_the_plain_one(d, P, kind, causal):
    """Held rows and attention for all heads of a sequence at once, against the ones an element
    and a query at a time."""
    rng = np.random.default_rng(3)
    lengths, counts, G, Hq, T = [150, 40, 0], [3, 2, 3], 2, 4, 3
    pool, table = H.filled(rng, 3, G, P, d, lengths)
    table = table.copy()
    table[0, 1] = -1
    q = torch.from_numpy(rng.standard_normal((3, Hq, T, d)))
    ref, tol = H.attend(pool, table, lengths, q, kind, counts, causal)
    tensors = pool.tensors("cpu")
    for b in range(3):
        held = H.held_rows(tensors, torch.from_numpy(table[b]), lengths[b])
        for g in range(G):
            for which, x in zip("kv", held[:2]):
                want = pool.rows(which, table[b], lengths[b], g)
                there = held[3].numpy()
                assert np.array_equal(there, ~np.isnan(want).any(1))
                assert np.array_equal(x[g].numpy()[there], want[there])
        out, t = H.attend_rows(held, q[b], counts[b], kind, causal)
        n = counts[b]
        # (float64: d + n additions, some 200 times 2^-53 of what is added, p |v|; a tolerance
        # has 2^-24 of that at least)
        assert (np.abs(out.numpy()[:, :n] - ref[b, :, :n]) <= 1e-5 * tol[b, :, :n]).all()
        assert np.allclose(t.numpy()[:, :n], tol[b, :, :n], rtol=1e-9, atol=1e-300)
