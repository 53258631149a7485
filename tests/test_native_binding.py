"""The compiled entry points are needed by the calls that go through them, and by nothing else."""
import os
import subprocess
import sys

_WITHOUT = """
import sys, types
import paper_2405_14371_b200 as package
from paper_2405_14371_b200 import build
build.build()
sys.modules["paper_2405_14371_b200._native_binding"] = None        # an import of it fails, as where it is missing or does not load
from paper_2405_14371_b200 import binding as B
import torch
assert package.Shard is B.Shard and B.es_version()
assert B.es_op_kv_plan_max_runs(4, 5, 16) == 5
import paper_2405_14371_b200.pipeline, paper_2405_14371_b200.stage
i, f, s = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 16, 64, dtype=torch.int8), torch.zeros(2, 2)
h = torch.zeros(2, 2, 64, dtype=torch.float16)
for call in (lambda: B.es_op_kv_plan(i, i, i.view(2, 1), 16, 4), lambda: B.es_op_kv8_append(h, h, i, f, f, s, s), lambda: B.es_op_kv8_gather(i, f, f, s, s),
             lambda: B.es_op_decode_attention_kv8(h, f, f, s, s, i.view(2, 1), i, 16), lambda: B.es_op_sample(s, s[0])):
    for _ in range(2):
        try:
            call()
        except ImportError as e:
            assert "_native_binding.so" in str(e) and "build" in str(e), e
        else:
            raise AssertionError("no refusal")
del sys.modules["paper_2405_14371_b200._native_binding"]
try:
    B.es_op_sample(s, s[0])
except B.EsError as e:
    assert e.status == 1
print("the rest works")
"""


def test_what_does_not_need_the_compiled_entry_points_works_without_them():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _WITHOUT], cwd=root, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "the rest works" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
