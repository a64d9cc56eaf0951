"""What the sources of the calls around a step have to keep to and no run shows."""
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


def test_the_rows_are_read_and_written_behind_the_wait_alone():
    # The kernel of the rows may start while the list's runs.  That the list's kernel has waited for the kernels before it tells the rows'
    # kernel nothing, so all that it reads and writes of global memory lies behind a wait of its own that every thread comes to.
    for kernel in ("rules_kernel", "rules_list_kernel"):
        body = _function(kernel, "rules_kernel.cuh")
        assert body.count("grid_dependency_sync();") == 1
        wait = body.index("grid_dependency_sync();")
        ahead, line = body[:wait], body[body.rindex("\n", 0, wait):body.index("\n", wait)].strip()
        assert line == "grid_dependency_sync();" and ahead.count("{") - ahead.count("}") == 1         # (under no condition)
        assert not re.search(r"__ldg|load_entry|load_granule|bulk_load|bulk_store|store_granule|atomic(?!Min\(&first_bad)|head\[|a\.status|rules_ends|rules_row\b", ahead)
        # no pointer of the arguments is followed
        assert not re.search(r"\ba\.\w+\[|[=(,;&|!]\s*\*\s*a\.|\b(?:in|out|signs)\[", ahead)


def test_the_rows_kernel_is_launched_only_behind_a_list_that_was():
    # A list whose launch failed is whatever the workspace held: the rows' kernel would follow its entries anywhere.
    body = _function("rules_call", "picospec_api.cu")
    at = body.index("e = launch_rules_list(")
    rest = body[at:]
    launches = list(re.finditer(r"launch_rules(?!_list)\b", rest))
    assert launches and not re.search(r"launch_rules(?!_list)\b", body[:at])
    for m in launches:
        assert rest[:m.start()].endswith("if (e == cudaSuccess) e = ")
    # (nothing in between takes the list's error away, and it is taken where it arises: one that stays is the next call's)
    assert not re.search(r"\be = ", rest[1:launches[0].start() - len("e = ")])
    assert "return cudaGetLastError();" in _function("launch_rules_list", "picospec_api.cu")


def test_gradients_are_scaled_only_behind_sums_that_were_taken():
    assert _function("grad_group", "picospec_api.cu").rstrip("}").rstrip().endswith("return cudaGetLastError();")
    assert re.search(r"for \(int i = 0; e == cudaSuccess && ", _function("grad_pass", "picospec_api.cu"))
    for name in ("picospec_grad_norm", "picospec_clip_grad"):
        body = _function(name, "picospec_api.cu")
        passes = list(re.finditer(r"grad_pass\(ctx, (false|true)", body))
        assert [m.group(1) for m in passes] == ["false", "true"]
        assert body[:passes[0].start()].endswith("e = ") and body[:passes[1].start()].endswith("if (e == cudaSuccess) e = ")
