"""What the library keeps between calls may be read and written by several threads at once: variables of that kind are atomic."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2206_07882_amd", "csrc")


def _plain_statics(text):
    """Static variables that are neither constant, nor atomic or a lock, nor of a thread's own."""
    text = re.sub(r"//[^\n]*", "", text)
    found = re.findall(r"\bstatic\s+(?!const\b|constexpr\b|inline\b|thread_local\b|std::atomic\b|std::mutex\b|__device__\b|_assert\b)[\w:<>, *&]+?\s*(?:\[[^;(){}]*\])*\s*(?:=[^;]*|\{[^;(){}]*\})?;", text)
    return [f for f in found if "(" not in f.split("=")[0]]


def test_state_between_calls_is_atomic():
    files = sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip")))
    assert len(files) > 10
    found = {os.path.basename(f): _plain_statics(open(f).read()) for f in files}
    assert not any(found.values()), {k: v for k, v in found.items() if v}


def test_the_search_finds_what_it_looks_for():
    for line in ("static bool allowed[QR_MAX_DEVICES];", "static int n = 0;", "static void *words;", "static unsigned seen{0};"):
        assert _plain_statics(line) == [line]
    for line in ("static std::atomic<bool> configured[QR_MAX_DEVICES];", "static const int n = 3;", "static constexpr int V = 4;", "static inline int f(int a);",
                 "static int small_n_max() { return 32; }", "static thread_local int n;", "static std::mutex one;", "static_assert(A % B == 0, \"\");"):
        assert not _plain_statics(line)
