"""Where the attention of include/tva_layer.h looks for positions whose pages were given back (entries below 0 in the page table): in the cache, whatever
the entry.  What a kernel reads there it drops, so that no result shows a read outside; the look-up itself is run on the host (CPU)."""
import os
import re
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_26577_amd", "csrc")


def test_places_of_pages_that_are_gone_lie_in_the_cache(tmp_path):
    exe = str(tmp_path / "cache_lookup")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--cuda-host-only", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "sanitize", "cache_lookup.hip"), "-o", exe], check=True)
    res = subprocess.run([exe], stdout=subprocess.PIPE, text=True, timeout=60)
    assert res.returncode == 0 and " 0 failure(s)" in res.stdout, res.stdout


def test_the_attention_looks_up_pages_in_no_other_way():
    source = open(os.path.join(CSRC, "chunk.hip")).read()
    assert re.findall(r"\bFinder<([^>]*)>", source) == ["PLACES != kDense, true"]
    assert not re.search(r"\btable\[|\bpage_table\[|\bposition_at\(", source)
