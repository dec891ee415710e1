"""Rules that the CUDA sources keep, checked on their text (no GPU needed)."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1904_02205_b200", "csrc")


def _sources():
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            yield name, re.sub(r"//[^\n]*", "", f.read())


def test_no_load_takes_the_read_only_path():
    """Kernels that start before their predecessor has ended may read what it writes only through ordinary loads:
    the compiler may move a read-only load above the wait."""
    for name, text in _sources():
        assert "__ldg(" not in text and "ld.global.nc" not in text, name
        hits = re.findall(r"const\s+\w+\s*\*\s*(?:const\s+)?__restrict__\s+\w+", text)
        assert not hits, "%s: %s" % (name, hits)


def test_limits_of_shared_memory_are_constants():
    """The limit belongs to a kernel on a device.  Host threads with contexts of their own share it: a call that set it to its own size
    could lower it between another thread's setting and launch."""
    texts = dict(_sources())
    number = r"[\d\s()*+uUlL]+"
    defined = {name: set(re.findall(r"const(?:expr)?\s+\w+\s+(\w+)\s*=\s*%s;" % number, t)) for name, t in texts.items()}
    shared = {n for names in defined.values() for n in names if re.match("k[A-Z]", n)}
    seen = 0
    for name, text in texts.items():
        constants = shared | defined[name]
        for size in re.findall(r"cudaFuncAttributeMaxDynamicSharedMemorySize\s*,\s*(?:\(int\)\s*)?([^;]*?)\)\s*(?:;|!=|\|\|)", text):
            seen += 1
            assert size in constants or re.fullmatch(number, size), "%s: %s" % (name, size)
    assert seen >= 5
