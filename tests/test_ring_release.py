"""A stage of a ring is given back by one lane for its warp, when every lane's loads have returned.  Where that lane's arrival stands
before the stores that use what was read, it has to depend on what ALL lanes have read: lanes may run apart, and then one lane's
loads have returned before another's.  A run hardly ever shows it, so the statements are checked in the sources."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2305_19982_b200" / "csrc"
VOTE = r"__any_sync\(0xffffffffu, \(.* & zero\) != 0u\)"


def _statements(name):
    text = re.sub(r"//[^\n]*", "", (CSRC / name).read_text())
    return [line.strip() for line in text.splitlines() if line.strip()]


def test_rows_of_logits():
    """Every arrival before the stores is given the outcome of a vote on what was read just before; the others stand behind
    a store of it."""
    lines = _statements("policy_loss.cu")
    begin = next(i for i, line in enumerate(lines) if line.startswith("const auto release = "))
    end = next(i for i in range(begin, len(lines)) if lines[i].startswith("decltype(row_mask(a, first)) next;"))
    body = lines[begin:end]
    assert any(re.match(r"const auto once_read = \[&\]\(unsigned read\) \{ return \(unsigned\)%s; \};$" % VOTE, line) for line in body)
    early = [i for i, line in enumerate(body) if line == "release(nothing);"]
    plain = [i for i, line in enumerate(body) if line.endswith("release();")]
    assert len(early) == 3 and len(plain) == 3 and not [line for line in body if re.search(r"release\((?!nothing\)|\))", line)]
    for i in early:
        vote = max(j for j in range(i) if body[j] == "const unsigned nothing = once_read(read);")
        assert body[vote - 1].startswith("for (int i = 0; i < ") and "read ^= u[i].x;" in body[vote - 1]
        assert not any("sh.stage" in line or "units[" in line for line in body[vote:i])
    # a row that nothing is written of is not read a second time; of the others a store comes first
    assert body[plain[0]].startswith("for (int at = 0; at < count;") and all("out.put" in " ".join(body[i - 3:i]) for i in plain[1:])


def test_8_bit_updates():
    lines = _statements("state8.cu")
    at = next(i for i, line in enumerate(lines) if "barrier_arrive(" in line and "+ nothing" in line)
    assert lines[at - 1] == "__syncwarp();" and re.match(r"const unsigned nothing = %s;$" % VOTE, lines[at - 2])
    assert all(part in lines[at - 2] for part in ("weights", "top.x", "top.y"))


def test_32_bit_updates():
    """Nothing is read of the stage behind the last store of what was read from it."""
    lines = _statements("fold_apply_multi.cu")
    at = next(i for i, line in enumerate(lines) if "barrier_arrive(" in line and "empty[" in line)
    begin = max(i for i in range(at) if "sh.stage[slot]" in lines[i])
    assert any("store4(" in line for line in lines[begin:at]) and not any("sh.stage" in line or "st.g" in line for line in lines[at:at + 25])
