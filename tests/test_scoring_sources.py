"""Rules of the scoring kernels that no run can show, checked on their source: copies into shared memory that do not come within the limit of a
wait, which no correct run reaches, leave numbers behind that are none."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_07899_b200", "csrc", "logits.cu")


def code():
    with open(SOURCE) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_every_wait_for_a_piece_is_asked_whether_it_came():
    calls = re.findall(r"[^\n]*\bpieces\.next\([^\n]*", code())
    assert len(calls) == 2
    for line in calls:
        assert re.search(r"if \(!pieces\.next\(.*\)\) run\.s = pair_of\(NAN, NAN\);|if \(!pieces\.next\(.*\)\) scale2 = pair_of\(NAN, NAN\);", line), line


def test_a_late_piece_of_the_gradient_shows_in_the_loss_of_whichever_cta():
    text = code()
    gradient = text[text.index("for (int i = i0; i - lead < row.hi; i += kBatch * kThreads) {", text.index("const f32x2 cc = ")):]
    gradient = gradient[:gradient.index("parity ^= 1;")]
    assert re.search(r"pmul\([^;]*, scale2\)", gradient)                   # what the gradient is multiplied by
    last = re.search(r"if \(([^;{}]*)\) g\.loss\[n\] = NAN;", gradient)
    assert last and "scale2" in last.group(1) and "rank" not in last.group(1)
