"""What the sources of the serving operators' kernels have to keep, where a run on the GPU would not show it reliably."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1909_00562_amd", "csrc")


def _kernel(name, file):
    """The text of a kernel, from its name to the closing brace."""
    with open(os.path.join(CSRC, file)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    at = text.index("{", re.search(r"__global__[^;{]*\b%s\(" % name, text).end())
    depth, end = 0, at
    while True:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
        if depth == 0:
            return text[at:end]


def test_single_shared_values_of_the_words_kernel_are_written_in_one_place():
    """A value in LDS that is written twice needs a barrier between the readers of the first and the second writer, also on the paths that
    leave steps out: the state of a sequence was overwritten by one wave while others might still have to read it."""
    body = _kernel("verify_words_kernel", "vocab_verify.hip")
    names = [n.strip() for decl in re.findall(r"__shared__ (?:int|double) ([^;]*);", body) for n in decl.split(",")]
    single = [n for n in names if "[" not in n]
    assert {"s_words", "s_n", "s_state", "s_last", "s_chunk", "s_theta"} <= set(single)
    for n in single:
        writes = re.findall(r"\b%s\s*=[^=]" % n, body)
        assert len(writes) == 1, (n, len(writes))


def test_no_order_of_memory_rests_on_a_wait_by_hand():
    """What blocks of one launch tell each other is ordered by atomics, or holds without an order: a wait for the chip's counters is none
    that the compiler knows of."""
    for file in ("vocab_verify.hip", "kv_attn.hip", "kv_cache.hip"):
        with open(os.path.join(CSRC, file)) as f:
            assert not re.search(r"s_waitcnt|signal_fence", re.sub(r"//[^\n]*", "", f.read())), file


def test_every_wait_for_other_blocks_ends():
    """A loop that reads what another block is to write counts its tries."""
    for file in ("vocab_verify.hip", "kv_attn.hip", "kv_cache.hip"):
        with open(os.path.join(CSRC, file)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for at in re.finditer(r"\bdo \{", text):
            body, condition = re.match(r"(.*?)\} while \(([^;]*)\);", text[at.end():], re.S).groups()
            if "__hip_atomic_load" in body:
                assert "++tries <" in condition, (file, condition)
        assert not re.search(r"while \([^;{]*__hip_atomic_load", text), file
