"""Stores to tensor memory are asynchronous: a thread that loads what it has stored waits for its stores first (waiting for loads is not enough).  The attention kernel
loads weights that it has made only to rescale them.  (Whether a load is too early is up to the hardware; the sources show the order.)"""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2605_02905_b200" / "csrc"


def test_weights_are_read_again_only_after_their_stores():
    code = re.sub(r"//[^\n]*", "", (CSRC / "eosq_kv8_attend_tc.cu").read_text())
    calls = [(m.start(), m.group(1)) for m in re.finditer(r"\b(tmem_(?:st|ld)(?:8|16|32|_wait))\(", code)]
    loads = [at for at, name in calls if name == "tmem_ld8"]
    assert loads   # weights, two to a column; scores and sums are read in sixteens and more
    for at in loads:
        stored = max(p for p, name in calls if name == "tmem_st8" and p < at)
        assert any(name == "tmem_st_wait" and stored < p < at for p, name in calls)
    # a tile's stores, sums among them, are waited for before the products are told that its weights are there
    told = code.index("mbar_arrive(&p_full[half])")
    last_store = max(p for p, name in calls if name in ("tmem_st8", "tmem_st16") and p < told)
    assert any(name == "tmem_st_wait" and last_store < p < told for p, name in calls)


def test_sums_are_rescaled_in_one_place():
    """A tile comes there once at most, so within a tile no load of a sum meets a store of the same."""
    code = re.sub(r"//[^\n]*", "", (CSRC / "eosq_kv8_attend_tc.cu").read_text())
    assert len(re.findall(r"\bmove\(", code)) == 1
    code = code[code.index("if (done < GROUPS)"):code.index("mbar_arrive(&p_full[half])")]
    before = code[:code.index("move(top)")]
    assert before.count("for (") == 1 and before.count("{") - before.count("}") == 2   # behind the look's loop, in no loop of the branch: the branch and the condition
