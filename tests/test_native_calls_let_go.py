"""Every native call into the library gives up the interpreter's lock (no GPU: read from the source): a launch may wait for room in the stream's queue, and other host
threads run meanwhile."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc", "marshal.cpp")


def test_every_call_that_launches_is_made_without_the_lock():
    code = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    names = re.findall(r"decltype\(&\w+\) (\w+);", code.split("struct Library {")[1].split("}")[0])
    launching = [n for n in names if not n.endswith("workspace_bytes")]
    assert len(launching) == 12
    runners = r"run\((?:[^;]|;(?! *\}))*?\[&\]\(const xconv_desc\* q, void\* ws, size_t n, void\* st\) \{\s*return $|unlocked\(\[&\] \{\s*return $|raise\(update\($"
    for n in launching:
        uses = [m.start() for m in re.finditer(r"\blib\.%s\b(?! *\|\|)" % n, code)]
        uses = [u for u in uses if not code[:u].endswith("!")]                  # (`!lib.forward`: whether the library is there)
        assert len(uses) == 1, n
        assert re.search(runners, code[max(0, uses[0] - 260):uses[0]]), n
    for body in (code.split("bool run(")[1].split("\n}\n")[0], code.split("xconv_status unlocked(")[1].split("\n}\n")[0]):
        at = re.search(r"\bs = call\(", body).start()
        assert body.index("Py_BEGIN_ALLOW_THREADS") < at < body.index("Py_END_ALLOW_THREADS")
    update = code.split("xconv_status update(")[1].split("\n}\n")[0]
    assert re.search(r"return unlocked\(\[&\] \{ return call\(", update)
