"""All sources of the library share a namespace, so a structure or a function with external linkage that two of them define
has to be one and the same: it belongs in a header."""
import collections
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2601_01473_amd", "csrc")
OWN_PROGRAMS = {"hbm_ceiling.hip"}


def _top_level(text):
    """The text of namespace scope: bodies of functions and structures as {}, no comments, no preprocessor lines."""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    text = re.sub(r"^[ \t]*#[^\n]*(\\\n[^\n]*)*", "", text, flags=re.M)
    text = re.sub(r'"(\\.|[^"\\])*"', '""', text)
    text = re.sub(r"namespace\s+\w+\s*\{|extern \"\"\s*\{", "", text)
    out, depth = [], 0
    for c in text:
        depth -= c == "}"
        if depth <= 0 or (c == "{" and depth == 0):
            out.append(c)
        depth += c == "{"
        depth = max(depth, 0)
    return re.sub(r"\{[^}]*\}", "{}", "".join(out))


def _types(parameters):
    """Parameter types without names and defaults."""
    parts, depth, last = [], 0, ""
    for c in parameters:
        depth += c in "<(["
        depth -= c in ">)]"
        if c == "," and depth == 0:
            parts.append(last)
            last = ""
        else:
            last += c
    types = []
    for p in parts + [last]:
        p = re.sub(r"=.*", "", p).replace("__restrict__", " ").strip()
        p = re.sub(r"(?<=[\s&*(>])\w+(?=\s*(\)?\s*\[[^\]]*\])?\s*$)", "", p)
        types.append(re.sub(r"\s+", "", p))
    return tuple(types)


def definitions(text):
    names = set()
    for m in re.finditer(r"([^;{}]*)\{\}", _top_level(text)):
        head = " ".join(m.group(1).split())
        inner = re.sub(r"__launch_bounds__\s*\((?:[^()]|\([^()]*\))*\)", "", head)
        inner = re.sub(r"template\s*<(?:[^<>]|<[^<>]*>)*>", "", inner).strip()
        kind = re.match(r"(?:struct|class|union|enum(?: class)?)\s+(?:__attribute__\s*\(\(.*?\)\)\s*)?(\w+)", inner)
        if kind:
            names.add(("structure", kind.group(1)))
            continue
        call = re.match(r"(.*?)\b(\w+)\s*\((.*)\)\s*(const|noexcept)?$", inner)
        if call and "static" not in call.group(1).split() and call.group(1).strip():
            names.add(("function", call.group(2)) + _types(call.group(3)))
    return names


def test_the_reader_of_definitions():
    text = """namespace agnes {
    struct A { int x; };  // struct B {}
    template <typename T, int N> __device__ __forceinline__ int f(const T* __restrict__ p, float (&x)[8], int64_t n = 3) { if (p) { return 1; } return 0; }
    static int g(int a) { return a; }
    __global__ __launch_bounds__(N == 3 ? 1 : 2) void k(A a) {}
    }"""
    assert definitions(text) == {("structure", "A"), ("function", "f", "constT*", "float(&)[8]", "int64_t"), ("function", "k", "A")}


def test_names_are_defined_once():
    where = collections.defaultdict(list)
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        if os.path.basename(path) not in OWN_PROGRAMS:
            with open(path) as f:
                for name in definitions(f.read()):
                    where[name].append(os.path.basename(path))
    assert len(where) > 200
    assert not {n: w for n, w in where.items() if len(w) > 1}
