"""Sort and weight gradient recorded into graphs: where their memory and curve tables come from (the host
layer against the stand-in for the HIP runtime of host_api.py, no GPU)."""
import host_api
from test_ops_routes import exe  # noqa: F401

SORT, DEPTH = "sort 9000 8 1 9000 0 {}", "depth 1700 2500 1024 0 4 {}"


def test_sort(exe):  # noqa: F811
    eager, _, rec, _, again, other = host_api.run(exe, [SORT.format(1), "capture 1 1", SORT.format(1), "capture 1 0", SORT.format(1),
                                                        SORT.format(2)])
    at = [dict(e)["sort"]["counts"] for e in (eager, rec, again, other)]
    assert at[0] == at[2] and len({at[0], at[1], at[3]}) == 3
    assert "malloc" in dict(rec) and "malloc_async" not in dict(rec) and "malloc_in_graph" not in dict(rec)


def test_weight_gradient_before_its_table_is_known(exe):  # noqa: F811
    _, rec, _, eager, again = host_api.run(exe, ["capture 1 1", DEPTH.format(1), "capture 1 0", DEPTH.format(1), DEPTH.format(2)])
    assert "order" in dict(rec) and dict(rec)["tile"]["table"] == dict(rec)["order"]["d"]      # the graph writes its own
    assert "order" in dict(eager) and dict(eager)["tile"]["table"] not in (0, dict(rec)["tile"]["table"])
    assert "order" not in dict(again) and dict(again)["tile"]["table"] == dict(eager)["tile"]["table"]


def test_weight_gradient_with_a_known_table(exe):  # noqa: F811
    first, second, _, rec, _ = host_api.run(exe, [DEPTH.format(1), DEPTH.format(2), "capture 2 1", DEPTH.format(2), "capture 2 0"])
    assert len({dict(e)["tile"]["table"] for e in (first, second, rec)}) == 1
    assert "order" in dict(first) and "order" not in dict(second) and "order" not in dict(rec)
