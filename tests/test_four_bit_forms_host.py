"""The GPU tests of the 4-bit products run every instance of their kernel that the library holds (no GPU needed: the launchers' rules over the tests' sizes)."""
import re

import pytest

import test_gpu_four_bit as G
import test_gpu_four_bit_forms as M
from four_bit_forms import Call, form_of
from test_kernel_resources import kernels  # noqa: F401


def sizes(test):
    """What a test is parametrised with, of its case."""
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize" and "," in m.args[0])


def reached():
    """(form, type of the result) -> the calls that run it."""
    found = {}

    def add(types, *call):
        if call[1]:                       # no rows: no launch
            for t in types:
                found.setdefault((call[0], form_of(Call(*call)), t), []).append(call)

    both, f32 = ("unsigned short", "float"), ("float",)
    for m, n, k in sizes(G.test_products_of_whole_numbers) + sizes(G.test_every_form_of_the_product):
        add(both, False, m, n, k)
    for counts, groups, n, k in sizes(G.test_grouped_products_of_whole_numbers):
        add(both, False, sum(counts) + 21, n, k, groups)
    for counts, n, k in sizes(G.test_every_form_of_the_grouped_product):
        add(f32, False, sum(counts) + 3, n, k, len(counts))
    for counts, n, k in sizes(M.test_sorted_products_of_whole_numbers):
        add(both, False, sum(counts) + 3, n, k, len(counts))
    for m, n, k in sizes(G.test_swiglu) + sizes(G.test_every_form_of_swiglu):
        add(both, True, m, n, k)
    for counts, n, k in sizes(G.test_every_form_of_grouped_swiglu):
        add(f32, True, sum(counts) + 3, n, k, len(counts))
    for counts, groups, n, k in sizes(G.test_grouped_swiglu):
        add(f32, True, sum(counts) + 5, n, k, groups)
    for rows, n, k in sizes(M.test_swiglu):
        if isinstance(rows, list):
            add(both, True, sum(rows) + 3, n, k, len(rows))
        else:
            add(both, True, rows, n, k)
    return found


def instances(kernels):  # noqa: F811
    """(swiglu, form, type) of every instance in the library."""
    found = set()
    for name in kernels:
        args = re.fullmatch(r"k_four_rows<(true|false), (.*), (float|unsigned short)>", name)
        if args:
            found.add((args.group(1) == "true", args.group(2), args.group(3)))
    return found


def test_every_instance_is_run(kernels):  # noqa: F811
    there, run = instances(kernels), set(reached())
    assert len(there) == 64 and run <= there
    assert not there - run


def test_sorted_rows_run_every_instance_but_those_for_dense_rows(kernels):  # noqa: F811
    """The tiles of 64 rows are not for sorted ones."""
    run = {key for key, calls in reached().items() if any(len(c) == 5 for c in calls)}
    assert {form.rsplit(", ", 2)[0] for _, form, _ in instances(kernels) - run} == {"8, 1, 4, 2, 1, 256, 2"}


@pytest.mark.parametrize("call,form", [
    ((False, 1, 7168, 2048), "1, 8, 1, 2, 1, 0, 2, true, true"), ((False, 2667, 2048, 768, 128), "4, 1, 2, 2, 1, 256, 3, true, true"),
    ((False, 173, 1543, 1440), "8, 1, 1, 1, 1, 1024, 4, false, false"), ((True, 3, 1408, 2048), "1, 8, 1, 1, 1, 0, 2, true, true"),
    ((True, 512, 2048, 7168, 32), "8, 1, 1, 1, 1, 512, 4, false, true")])
def test_forms_that_a_profiler_saw(call, form):
    assert form_of(Call(*call)) == form
