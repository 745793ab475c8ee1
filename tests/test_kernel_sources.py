"""Rules of the kernel sources that no run on a GPU shows reliably."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2401_16757_gb300", "csrc")
WEIGHTS = {"W", "g", "table"}  # parameters that hold weights (g: RMSNorm gains; table: the embedding's)


def _kernels():
    """(file, head, body) of every kernel that starts before the launch ahead of it has ended."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__", text):
            start = text.index("{", m.end())
            end = text.index("\n}", start)
            if "pdl_wait()" in text[start:end]:
                yield os.path.basename(path), text[m.end():start], text[start:end]


def test_outputs_of_an_overlapped_launch_are_not_read_as_read_only():
    """A read-only load (ld.global.nc) is for memory that nothing writes while the kernel runs, and may be moved across
    the wait for the launch before, which is still writing this kernel's inputs when it starts."""
    seen = 0
    for name, head, body in _kernels():
        seen += 1
        assert "__ldg(" not in body, (name, head)
        params = re.findall(r"const\s+\w+\s*\*\s*__restrict__\s+(\w+)", head)
        assert set(params) <= WEIGHTS, (name, params)
    assert seen >= 18


def test_rotation_releases_the_attention_after_its_wait():
    """The attention kernels read the position and older cache rows before their own wait: what they overlap, the
    rotation launched right before them, lets them start only once everything ahead of it has ended."""
    bodies = [body for _, head, body in _kernels() if "rope_append_kernel" in head]
    assert len(bodies) == 1
    assert 0 <= bodies[0].index("pdl_wait()") < bodies[0].index("pdl_launch_dependents()")
    assert not re.search(r"\breturn\b", bodies[0][:bodies[0].index("pdl_launch_dependents()")])
    text = open(os.path.join(CSRC, "k_decoder.cu")).read()
    launch = text[text.index("int launch_attention("):]
    between = launch[launch.index("rope_append_kernel<T, 1, 1>"):launch.index("attention_split_kernel<T>, static_cast")]
    assert between.count("launch_pdl(") == 0 and between.count("launch_attention_tc(") == 1


def _text(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def test_no_wait_for_a_phase_while_the_one_before_may_be_open():
    """A parity wait for phase g returns at once while phase g - 1 is still open.  The products of a half complete its
    o_full phase tile by tile; a softmax warp that did not wait for phase g - 1 waits for it before it waits for phase g."""
    body = next(body for _, head, body in _kernels() if "attention_rows_kernel" in head)
    waits = list(re.finditer(r"mbar_wait_bounded\(o_full\(half\), (\(g - 1\) & 1|g & 1)", body))
    assert waits
    for i, w in enumerate(waits):
        if w.group(1) == "g & 1":
            assert i > 0 and waits[i - 1].group(1) == "(g - 1) & 1"
            between = body[waits[i - 1].end():w.start()]
            assert ";" not in between and "{" not in between  # one condition: the first has to hold for the second


def test_outputs_in_tensor_memory_pass_a_fenced_barrier_between_the_halves():
    """A softmax warp may have changed its half's outputs in tensor memory by hand; the other half's warps read them behind
    a barrier, which orders tensor memory only with a fence on either side."""
    body = next(body for _, head, body in _kernels() if "attention_rows_kernel" in head)
    at = body.index("ml[half * 128 + slot] = make_float2(m, l);")
    behind = body[at:body.index("tmem_ld_32x32b_x32", at)]
    barrier = re.search(r"if \(REP == 1\) row_sync\(\); else all_sync\(\);", behind)
    assert "tc_fence_before()" in behind[:barrier.start()] and "tc_fence_after()" in behind[barrier.end():]


def test_dependents_start_only_once_a_kernel_holds_its_tensor_memory():
    """Tensor memory is allocated by waiting until an SM has enough of it.  A kernel launched behind another may start as soon
    as that one's CTAs have released it, and may then hold tensor memory while it waits for that one's end: a CTA that
    releases it before its own allocation could wait for that memory for ever."""
    seen = 0
    for name, head, body in _kernels():
        if "tmem_alloc(" not in body or "pdl_launch_dependents()" not in body:
            continue
        seen += 1
        assert body.index("tmem_alloc(") < body.index("= *tmem_slot;") < body.index("pdl_launch_dependents()"), (name, head)
        between = body[body.index("tmem_alloc("):body.index("= *tmem_slot;")]
        assert "__syncthreads()" in between, (name, head)
    assert seen >= 6
