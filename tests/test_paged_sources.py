"""Orders in the paged attention kernels that no run can show to be missing (a CTA
would have to be held up for seconds at the wrong place), read from the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_04185_gb300", "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def _body(text, name):
    """The braces behind the definition of function `name`."""
    at = re.search(name + r"\([^;{]*\)\s*\{", text).end()
    depth, end = 1, at
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[at:end]


def _in_order(text, *parts):
    at = -1
    for p in parts:
        at = text.find(p, at + 1)
        assert at >= 0, p


def test_no_cta_of_a_cluster_ends_before_all_have_pushed():
    """Stores into a CTA that has ended are not allowed, whatever its waits came to."""
    merge = _body(_code("paged_tc.cuh"), "merge_in_cluster")
    _in_order(merge, "cluster_arrive()", "mbar_wait(merge_bar", "if (come) merge_rows", "cluster_wait()",
              "if (!come) mbar_wait(merge_bar")
    assert "return" not in merge
    for name, kernel in (("paged_attention_tc.cu", "paged_tc_kernel"), ("paged_attention_rows.cu", "paged_rows_kernel")):
        body = _body(_code(name), kernel)
        pushes = [m.start() for m in re.finditer(r"\bst_async\(", body)]
        assert pushes and body.count("merge_in_cluster") == 1 and body.index("merge_in_cluster") > max(pushes)
        assert not re.search(r"\bmerge_rows\b|mbar_wait\(&merge_bar", body)
        # the only early end is that of a CTA without a cluster
        assert re.findall(r"[^;{}]*\breturn;", body[body.index("tc_dealloc"):]) == ["\n  if (a.splits == 1) return;"]


def test_dependents_start_only_where_tensor_memory_is_taken():
    """The kernel that follows may take tensor memory before it waits for this grid."""
    for name, kernel in (("paged_attention_tc.cu", "paged_tc_kernel"), ("paged_attention_rows.cu", "paged_rows_kernel")):
        body = _body(_code(name), kernel)
        conditions = [x.strip() for x in re.findall(r"([^;{}]*)grid_dependents_launch\(\);", body)]
        assert conditions == ["if (n == 0)", "if (n > 0 && ok)"]
        _in_order(body, "tc_alloc(", "if (n == 0) grid_dependents_launch();")
