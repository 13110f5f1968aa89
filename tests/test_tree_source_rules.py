"""Rules that the kernels of a speculative step keep and no run can show."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_16213_gb300", "csrc")


def closing(code, i, pair):
    """The place behind what closes the bracket before place i."""
    depth = 1
    while depth:
        depth += {pair[0]: 1, pair[1]: -1}.get(code[i], 0)
        i += 1
    return i


def loops(code):
    """The bodies of the loops of `code` that have braces."""
    for m in re.finditer(r"\bfor \(", code):
        head = closing(code, m.end(), "()")
        if code[head:].lstrip().startswith("{"):
            start = code.index("{", head) + 1
            yield code[start:closing(code, start, "{}") - 1]


def test_loads_from_tensor_memory_are_the_whole_warps():
    """tcgen05.ld and its wait want every lane of the warp at the same instruction.  So no lane leaves an iteration of
    their loops early, and a loop whose lanes may part gathers them before the next iteration."""
    code = re.sub(r"//.*", "", open(os.path.join(CSRC, "tree_attn_tc.cu")).read())
    bodies = [b for b in loops(code) if re.search(r"tmem_ld\d+_issue\(", b) and not any(
        re.search(r"tmem_ld\d+_issue\(", inner) for inner in loops(b))]
    assert len(bodies) >= 2
    for b in bodies:
        assert "continue;" not in b and "break;" not in b, b
        if re.search(r"\bif \(", b):
            assert b.rstrip().endswith("__syncwarp();"), b


def test_the_walks_words_are_written_behind_their_readers():
    """The walking warp's lanes read the last round's words (A among them); the lane that writes the next round's waits for them."""
    code = re.sub(r"//.*", "", open(os.path.join(CSRC, "tree_verify.cu")).read())
    writes = [m.start() for m in re.finditer(r"if \(tid == 0\) \{\s*sm->node = ", code)]
    assert len(writes) == 1
    for w in writes:
        assert code[:w].rstrip().endswith("__syncwarp();")


def test_rotary_counts_tokens_past_an_int():
    """Up to 2^31 - 1 tokens: the last CTA's places behind them, and their number rounded up, do not fit an int."""
    code = re.sub(r"//.*", "", open(os.path.join(CSRC, "rotary.cu")).read())
    assert re.findall(r"(\S+ \S+) = blockIdx.x \* tokens", code) == ["uint32_t t"] and "t >= (uint32_t)a.T" in code
    assert re.findall(r"(\S+) \+ tokens - 1", code) == ["((int64_t)a.T"]


def test_the_largest_vocabulary_is_said_once():
    """The check of the argument and the shared memory that it keeps from overflowing go by one number."""
    said = [name for name in sorted(os.listdir(CSRC)) for _ in re.findall(r"\bkMaxVocab =", open(os.path.join(CSRC, name)).read())]
    assert said == ["tree.cuh"]
