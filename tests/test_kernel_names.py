"""Names in the kernels' sources (CPU)."""
import collections
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_10402_amd", "csrc")


def test_a_type_has_one_definition():
    """The .hip files share one namespace and become one library, so a struct of one file's own whose name
    another file gives to something else would be two types under one name."""
    found = collections.defaultdict(set)
    for name in os.listdir(CSRC):
        text = open(os.path.join(CSRC, name)).read()
        text = re.sub(r"^namespace \{$.*?^\}  // namespace$", "", text, flags=re.M | re.S)  # (names of the file alone)
        for m in re.finditer(r"^(?:template <[^>]*>\s*)?(?:struct|class|union|enum) (\w+)[^;{]*\{", text, re.M):
            found[m.group(1)].add(name)
    assert len(found) > 30
    assert {k: sorted(v) for k, v in found.items() if len(v) > 1} == {}
