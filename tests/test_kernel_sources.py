"""What the sources of the kernels have to keep to and no run shows."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_19133_b200", "csrc")


def _function(name, file):
    """The body of a function of a source file, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, file)).read())
    at = text.index("{", re.search(r"\b%s\(" % name, text).start())
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]
    raise AssertionError("unbalanced")


def test_no_cta_of_a_sampling_cluster_ends_while_a_peer_may_read_its_memory():
    # Remote shared memory is there for as long as its CTA runs.  The passes behind the statistics end with reads of it, so a CTA arrives at
    # the cluster's barrier behind the last of them, and waits for the others before it ends.
    # With limits that is find_cut; without, the sums that decide a draw on a border, if they were taken (row.exact).
    body = _function("sample_kernel", "sample_kernel.cuh")
    remote = r"peer_|_pass\(|take_total|gather|number|exact_total|find_cut"
    cut, limited = body.index("find_cut"), body.index("cluster_arrive();", body.index("find_cut"))
    plain = body.index("const bool asked = limited || row.exact;")
    assert "if (!limited && row.exact) cluster_arrive();" in body[plain:]
    assert body.rindex("if (limited) {", 0, cut) > 0 and body[limited:].split()[1] == "}" and limited < plain
    assert "return;" not in body[cut:plain] and body.count("cluster_arrive();") == 3      # (one more at the start)
    assert "exact = true;" in _function("take_total", "sample_kernel.cuh")
    draw = re.sub(r"if \(guard > 0\.0 &&.*?continue;\s*\}", "", body[limited:plain], flags=re.S)
    assert "guard = limited ||" in draw
    assert not re.search(remote, draw) and not re.search(remote, body[plain:])
    ends = [m.start() for m in re.finditer(r"return;", body[plain:])] + [body[plain:].rindex("}")]
    assert len(ends) == 2 and all(body[plain:][:e].rstrip().endswith("if (asked) cluster_wait();") for e in ends)


def test_a_wait_has_one_outcome_for_a_warp():
    # Lanes poll a barrier by themselves and may differ; what they tell the CTAs of the cluster may not.
    for kernel, file in (("sample_kernel", "sample_kernel.cuh"), ("distill_kernel", "distill_kernel.cuh")):
        body = _function(kernel, file)
        told = body.index("peer_store(peer_addr(")
        assert re.search(r"late = __reduce_max_sync\(", body[:told]), kernel


def test_a_cut_counts_ties_that_a_pass_has_counted():
    # A cut that is not `listed` (its last word) has level 1 read the numbers of ties per chunk, which a pass has to have written.
    body = _function("find_cut", "sample_kernel.cuh")
    cuts = list(re.finditer(r"return SampleCut\{([^}]*)\}", body))
    assert len(cuts) >= 4
    for m in cuts:
        if m.group(1).split(",")[-1].strip() != "true":
            counted = body.rfind("ties_at = row.mass_pass(", 0, m.start())
            assert counted >= 0 and not re.search(r"return SampleCut|continue;", body[counted:m.start()]), m.group(0)
