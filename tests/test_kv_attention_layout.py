"""The attention kernels' barriers, as they are laid out one behind the other, against the number their shared memory is checked for."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2307_09782_b200", "csrc")


def names(slots, **kw):
    return dict(C_kKeySlots=slots[0], C_kValueSlots=slots[1], **kw)


@pytest.mark.parametrize("source,last,values", [
    ("kv_attention_few.cu", "drain", [names((9, 9), kSegs=4), names((3, 2), kSegs=4)]),
    ("kv_attention_rows.cu", "drain", [names((3, 2), kSegs=4, kScaleSlots=4), names((2, 2), kSegs=4, kScaleSlots=4)]),
])
def test_barriers_are_counted(source, last, values):
    text = open(os.path.join(CSRC, source)).read()
    steps = re.findall(r"uint64_t\* (\w+) = (\w+)(?: \+ ([\w:]+))?;", text)
    steps = steps[[s[0] for s in steps].index("k_full"):]
    steps = steps[:[s[0] for s in steps].index(last) + 1]
    count = re.search(r"kNumBars = ([^;]+);", text).group(1)
    size = 2 if re.search(r"drain;\s+// \[2\]", text) or re.search(rf"{last} = \w+ \+ \w+;\s+// \[2\]", text) else 1
    for v in values:
        def number(e):
            return int(eval(e.replace("C::", "C_"), {}, v))
        at = {"bar": 0}
        for name, base, by in steps:
            at[name] = at[base] + (number(by) if by else 0)
        total = eval(re.sub(r"\bk(Key|Value)Slots", r"C_k\1Slots", count), {}, v)
        assert at[last] + size == total, (at, total)
