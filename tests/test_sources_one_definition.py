"""Types of one name in one namespace are one type: what two source files define apart from each other is in an unnamed namespace, or has two names."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc")


def types_of(code):
    """Names of the structs and classes that a source file defines with external linkage, with their namespaces."""
    code = re.sub(r"//[^\n]*|/\*.*?\*/", "", code, flags=re.S)
    code = re.sub(r'"(?:\\.|[^"\\\n])*"', '""', code)
    code = re.sub(r"^\s*#(?:[^\n]*\\\n)*[^\n]*", "", code, flags=re.M)
    found, scopes = [], []                                         # scopes: a namespace's name ("" unnamed), or None for any other brace
    for m in re.finditer(r"\bnamespace\s*(\w*)\s*\{|\b(template\s*<[^;{}]*>\s*)?(?:struct|class)\s+(?:alignas\([^)]*\)\s*)?(\w+)(\s*(?::(?!:)[^{;()]*)?)\{|\{|\}", code):
        text = m[0]
        if text == "}":
            scopes.pop()
        elif text.startswith("namespace"):
            scopes.append(m[1])
        else:
            if m[3] and None not in scopes and "" not in scopes:
                found.append("::".join([*scopes, m[3]]))
            scopes.append(None)
    assert not scopes
    return found


def test_the_reader_of_sources():
    code = """
    struct A { int x; };            // } struct B {
    namespace n { struct A { struct Inner {}; }; namespace { struct A {}; } template <typename T> struct C : A { void f() { struct D {}; } }; class E;
    inline void g(struct A* a) { } enum F { G }; }
    """
    assert types_of(code) == ["A", "n::A", "n::C"]


def test_no_two_types_of_one_name():
    where = {}
    for top, _, names in os.walk(CSRC):
        for name in names:
            if name.endswith((".cu", ".cuh", ".h", ".cpp")):
                for t in types_of(open(os.path.join(top, name)).read()):
                    where.setdefault(t, []).append(os.path.relpath(os.path.join(top, name), CSRC))
    assert len(where) > 20
    assert not {t: files for t, files in where.items() if len(files) > 1}
