"""How an attention call is cut into workgroups (serve_validate.cpp's attend_plan), without a
GPU: the calls of _serve_variants.py take the kernels that they are there for, and plans of
random calls, the largest sizes together among them, are what the kernels assume."""
import os
import shutil
import subprocess

import pytest

import _serve_variants as V

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_23253_amd", "csrc")
DTYPES = {"f32": 0, "bf16": 1, "f16": 2}


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """The program's answers: a dict of every call's plan, and its last line."""
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = tmp_path_factory.mktemp("plan") / "serve_plan"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
           os.path.join(ROOT, "tests", "native", "serve_plan.cpp"),
           os.path.join(CSRC, "serve_validate.cpp"), os.path.join(CSRC, "e2s_validate.cpp"),
           "-o", str(exe)]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    lines = []
    for c in V.CALLS.values():
        lines.append(" ".join(str(x) for x in (
            1 << 16, c["page"], c["kv_heads"], c["head_dim"], c["batch"], c["heads"], c["queries"],
            DTYPES[c["dtype"]], c["max_tokens"], int(c.get("causal", True)),
            int(c.get("weights", False)))))
    run = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True,
                         timeout=300)
    said = [x.split()[1:] for x in run.stdout.splitlines() if x.startswith("plan ")]
    names = ("status", "shared_rows", "tiles", "waves", "lse_kept", "splits", "chunk", "bytes")
    return dict(zip(V.CALLS, (dict(zip(names, map(int, x))) for x in said))), run


def test_plans_hold_together(plans):
    _, run = plans
    assert run.returncode == 0 and " 0 failures" in run.stdout, run.stdout[-2000:] + run.stderr


@pytest.mark.parametrize("name", V.CALLS)
def test_calls_take_their_kernels(plans, name):
    p, c = plans[0][name], V.CALLS[name]
    assert p["status"] == 0
    for key, want in c["plan"].items():
        if key == "few_parts":           # joined by join_few or join_many
            assert (1 < p["splits"] <= 8) if want else p["splits"] > 8, p
        elif key == "steps":             # of 64 keys, of a workgroup that parts the rows
            assert min(p["chunk"], max(V.lengths_of(c))) // 64 > want, p
        elif key == "quarter":           # keys of a wave
            assert p["chunk"] // p["waves"] > want and max(V.lengths_of(c)) > want, p
        else:
            assert p[key] == want, (key, p)


def test_every_kernel_is_taken():
    """Each instance of the main kernels' shapes that the dispatch has, and each way to join
    and to add up weights, is some call's."""
    def has(**kw):
        return any(all(c["plan"].get(k, c.get(k)) == v for k, v in kw.items())
                   for c in V.CALLS.values())
    for shared, tiles, waves in ((1, 1, 4), (1, 2, 4), (0, 1, 4), (0, 2, 4), (0, 1, 8), (0, 2, 8)):
        assert has(shared_rows=shared, tiles=tiles, waves=waves)
        assert has(shared_rows=shared, tiles=tiles, waves=waves, head_dim=128)
    for d in (64, 128):
        assert has(lse_kept=1, shared_rows=0, head_dim=d)
        assert has(few_parts=0, head_dim=d)
    assert has(few_parts=1, shared_rows=1) and has(few_parts=1, shared_rows=0)
