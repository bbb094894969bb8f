"""The stores of large results keep their hint through the compiler: kernels made for them store past the caches, the others do not."""
import functools
import importlib.util
import os
import re
import subprocess
import tempfile

import pytest

from conftest import ROOT

spec = importlib.util.spec_from_file_location("hip_build", os.path.join(ROOT, "paper_2404_09544_amd", "build.py"))
build = importlib.util.module_from_spec(spec)
spec.loader.exec_module(build)


@functools.lru_cache(maxsize=None)
def assembly(source):
    try:
        hipcc = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    with tempfile.TemporaryDirectory() as tmp:
        out = os.path.join(tmp, "code.s")
        r = subprocess.run([hipcc, *build.FLAGS, "-w", "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", out],
                           capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
        with open(out) as f:
            return f.read()


@pytest.mark.parametrize("source,kernel", [("embedding.hip", "k_embedding"), ("embedding.hip", "k_embedding_grad"), ("clip.hip", "k_clip")])
def test_hint_reaches_the_code(source, kernel):
    text = assembly(source)
    seen = {True: 0, False: 0}
    # the last template argument: Lb1 for the kernel of large results
    for name, streamed in re.findall(r"^(_ZN5gnnav\d+%sI\w*?Lb([01])EEEv\w*):" % kernel, text, re.M):
        body = text[text.index("\n" + name + ":"):]
        wide = re.findall(r"global_store_dwordx4 .*", body[:body.index(".Lfunc_end")])
        if kernel == "k_clip" and not wide:
            continue   # (the norm alone)
        assert any(re.search(r"\bnt\b", w) for w in wide) == (streamed == "1"), name
        seen[streamed == "1"] += 1
    assert seen[True] > 1 and seen[False] > 1, seen
