"""GPU tests that the pool's check() sees the device errors of every call of a serving step, and that the README's lines are
such calls."""
import os
import re

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__ as g
    g.build()
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def names():
    """What the README's serving lines work on: two requests of 40 and 20 tokens in pages of 16."""
    from paper_2609_38706_gb300.service import KVPages
    kv = KVPages(8, 16, 2, 64)
    x = lambda n, h: torch.randn((n, h, 64), device="cuda").to(torch.bfloat16)
    off = dev(np.array([0, 40, 60]))
    return dict(kv=kv, q=x(60, 4), k=x(60, 2), v=x(60, 2), q_off=off, k_off=off.clone(), tok_off=off.clone(), n_tokens=60,
                start=dev(np.zeros(2, np.int32)), pages=dev(np.arange(6, dtype=np.int32).reshape(2, 3)), k_new=x(60, 2),
                v_new=x(60, 2), kv_len=dev(np.array([40, 20], np.int32)), weight=torch.zeros((2, 3), device="cuda"))


def block():
    text = open(os.path.join(ROOT, "README.md")).read()
    return next(b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "kv = KVPages(" in b)


def lines():
    body = block()[block().index("kv = KVPages("):].split("\n")[1:]
    return [x.split("#")[0].strip() for x in body if x.strip()]


def run(line, env):
    if line.startswith("out, lse = kv.attend("):
        env = dict(env, q=env["q"][:2].unsqueeze(1))
    if "budget=64" in line:
        line = line.replace("budget=64", "budget=2").replace("recent=4", "recent=1")
    scope = {}
    exec(block()[:block().index("kv = KVPages(")], scope)  # its imports
    exec(line, scope, env)


def test_the_readmes_lines_run_and_check_nothing_wrong():
    env = names()
    assert len(lines()) == 6 and lines()[-1] == "kv.check()"
    for line in lines():
        run(line, env)


@pytest.mark.parametrize("call,name,value", [
    ("kv.read(", "tok_off", [0, 99, 60]), ("attend_prompt(", "q_off", [0, 99, 60]), ("attend_prompt(", "k_off", [-1, 40, 60]),
    ("kv.write(", "start", [0, -5]), ("kv.attend(", "kv_len", [40, 99]), ("evict", "kv_len", [-2, 20]),
])
def test_check_sees_the_error_of_each_call(call, name, value):
    from paper_2609_38706_gb300 import pk
    env = names()
    line = next(x for x in lines() if call in x)
    run(line, dict(env))
    env["kv"].check()
    env[name] = torch.tensor(value, dtype=env[name].dtype, device="cuda")
    run(line, env)
    with pytest.raises(pk.PKError):
        env["kv"].check()
