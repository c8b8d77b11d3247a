"""Which kernel a call of attention over the 4-bit cache goes to: the plan's own checks, that the GPU tests' calls reach the
kernels that they are meant for, and the registers that the plan's counts of resident blocks rest on."""
import ast
import ctypes
import os
import re
import subprocess

import pytest

from paper_2509_21009_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = os.path.join(ROOT, "tests", "cpp", "kvq_plan.cpp")
CSRC = os.path.join(ROOT, "paper_2509_21009_amd", "csrc")


def test_plan_under_sanitizers(tmp_path):
    """Every column is one kernel's, items and grids are within their limits, and an engine's workspace holds what any of its
    calls asks for."""
    exe = tmp_path / "kvq_plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", f"-I{CSRC}",
                    SOURCE, "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "plan tests passed" in r.stdout, r.stderr


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = tmp_path_factory.mktemp("plan") / "kvq_plan.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{CSRC}", SOURCE, "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))

    def call(n_q, n_kv, hd, ctx, rows, kind, bf16=True):
        """The plan of a test's call: its sequences' sizes, or the bounds that `kind` puts in their place."""
        room = _from_gpu_tests("test_gpu_kvq.py", "_room")(kind, n_q, hd)
        rows = [1] * len(ctx) if rows is None else rows
        n_rows, max_rows, tokens = sum(rows), max(rows), max(64, *(-(-c // 64) * 64 for c in ctx))
        if room:
            n_rows = max_rows = max(room[0], n_rows)
            tokens = max(tokens, room[1] // 64 * 64)
        out = (ctypes.c_int * 6)()
        lib.kvq_plan_of(n_q, n_kv, hd, int(bf16), len(ctx), n_rows, max_rows, tokens, 1, out)
        return dict(zip(("prompt_tiles", "prompt_waves", "prompt_items", "walk_tiles", "waves", "items"), out))

    return call


def _from_gpu_tests(file, name):
    """A function or constant of a test file that cannot be imported without a GPU."""
    tree = ast.parse(open(os.path.join(ROOT, "tests", file)).read())
    for node in tree.body:
        if isinstance(node, ast.FunctionDef) and node.name == name or \
                isinstance(node, ast.Assign) and getattr(node.targets[0], "id", None) == name:
            scope = {}
            exec(compile(ast.Module([node], []), file, "exec"), scope)
            return scope[name]
    raise KeyError(name)


PROMPT = {"tiles": (4, 1), "split": (4, 2), "eight": (8, 1)}  # waves; items: one, or two at least


def _takes_prompts(p, kind):
    waves, items = PROMPT[kind]
    return p["prompt_tiles"] > 0 and p["prompt_waves"] == waves and (p["prompt_items"] == 1 if items == 1 else p["prompt_items"] >= items)


@pytest.mark.parametrize("n_q,n_kv,hd,kinds", [
    (28, 4, 128, "tiles split eight"), (14, 2, 64, "tiles split"), (40, 2, 128, "split eight"), (3, 3, 64, "tiles"),
    (3, 1, 128, "eight"), (6, 1, 64, "split"), (6, 2, 64, "tiles split"), (6, 2, 128, "tiles split eight"),
    (7, 1, 128, "tiles split eight"), (7, 1, 64, "tiles split")])
def test_bounds_steer_prompts_to_their_kernel(plan, n_q, n_kv, hd, kinds):
    """The bounds that stand for a kind of call, at every head layout that a GPU test uses them with, for a few sequences and (but
    for split tiles, which are few) many."""
    for kind in kinds.split():
        for ctx, rows in (([1, 70], [1, 70]), ([1200, 300, 64, 5, 200], [100, 80, 64, 1, 20]), ([130] * 150, [20] * 150))[:2 if kind == "split" else 3]:
            assert _takes_prompts(plan(n_q, n_kv, hd, ctx, rows, kind), kind), (kind, plan(n_q, n_kv, hd, ctx, rows, kind))


def test_softmax_forms_go_to_their_kernels(plan):
    want = {"four": (4, 1), "four-64": (4, 1), "one": (1, 1), "eight-waves": (8, 1), "joined": (4, 2), "joined-64": (4, 2)}
    forms = _from_gpu_tests("test_gpu_kvq_softmax.py", "FORMS")
    for name, form in forms.items():
        p = plan(*form)
        if name.startswith("prompt"):
            assert _takes_prompts(p, form[-1]), (name, p)
            continue
        waves, items = want[name]
        for bf16 in (True, False):
            p = plan(*form, bf16)
            assert p["prompt_tiles"] == 0 and p["waves"] == waves and (p["items"] == 1 if items == 1 else p["items"] >= 2), (name, p)


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc")
def test_registers_and_scratch():
    """No kernel spills, and the waves of a SIMD are those that the plan counts with: attention's blocks of four waves three to
    a compute unit (two in fp32 at 128 dims), k_kvq_prompt's two."""
    asm = subprocess.run([build.HIPCC, *build.COMMON, *build.DEVICE, "--cuda-device-only", "-S", os.path.join(build.CSRC, "k_kvq.hip"),
                          "-o", "-"], check=True, capture_output=True, text=True, timeout=300).stdout
    info = {m.group(1): (int(m.group(2)), int(m.group(3))) for m in
            re.finditer(r"^(_Z\w+):.*?; TotalNumVgprs: (\d+).*?; ScratchSize: (\d+)", asm, flags=re.S | re.M)}
    assert len(info) > 40 and not [k for k, (_, scratch) in info.items() if scratch]
    for name, most in (("k_kvq_promptILi128ELi4E", 256), ("k_kvq_promptILi128ELi8E", 256), ("k_kvq_promptILi64ELi4E", 256),
                       ("k_kvq_attendILi128ELb0ELi4E", 168), ("k_kvq_attendILi64ELb0ELi4E", 128), ("k_kvq_attendILi128ELb1ELi4E", 256),
                       ("k_kvq_attendILi64ELb1ELi4E", 128)):
        found = [v for k, (v, _) in info.items() if name in k]
        assert len(found) == 1 and found[0] <= most, (name, found)
