"""What the library keeps on the host between calls: several threads call it at once (the binding releases the
interpreter's lock), so what one writes and another reads is atomic, or constant, or a thread's own."""
import glob
import os
import re
import threading

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_kept_variables_are_atomic():
    csrc = os.path.join(ROOT, "paper_2601_08670_gb300", "csrc")
    files = [f for e in ("cu", "cuh", "cpp") for f in glob.glob(os.path.join(csrc, "*." + e))]
    assert len(files) > 15
    kept = {}
    for path in files:
        src = re.sub(r"//[^\n]*", "", open(path).read())
        # variables, not functions or members that are constants
        for line in re.findall(r"^\s*static\s+[^()=;{]*?\w+\s*(?:\[[^;]*?\])*\s*(?:=[^;]*|\{[^;]*\})?;", src, re.M):
            kept.setdefault(os.path.basename(path), []).append(" ".join(line.split()))
    assert {"host.cu", "sample.cuh", "paged_attention.cuh"} <= set(kept)
    plain = [(f, v) for f, vs in kept.items() for v in vs if not re.match(r"static (constexpr|const|thread_local|std::atomic<) ?", v)]
    assert plain == []


def test_errors_are_each_threads_own():
    from paper_2601_08670_gb300 import build
    build.build()
    import paper_2601_08670_gb300 as pced
    L, bad = pced.lib(), []

    def call(i):
        for _ in range(2000):
            rc = L.pced_sample(4096, 0, 100, 2, 100, 4096, None, None, None, None, 4096 + 4 * (i == 0) - 2, None, None, None)
            if rc != 1:
                bad.append(rc)
    threads = [threading.Thread(target=call, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
