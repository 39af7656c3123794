"""Order of the barriers of attention behind shared prefixes: a phase is never passed over (host model of the waits)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PLANNED = 4      # segments that are planned ahead


@pytest.fixture(scope="module")
def units_of(tmp_path_factory):
    """Units that a group has of a segment, by the kernels' own rule compiled for the host."""
    d = tmp_path_factory.mktemp("order")
    src, lib = d / "x.cpp", d / "x.so"
    src.write_text('#include "%s/paper_2504_08791_b200/csrc/paged_index.h"\n'
                   'extern "C" int units_of(int both, int n, int group) { return prima::prefix_group_units(both != 0, n, group); }\n' % ROOT)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    return ctypes.CDLL(str(lib)).units_of


def unordered(segments, takes_part, units_of):
    """Pairs of phases of a group's query barrier of which the later one may complete before the earlier one has been waited
    for.  Events and what orders them: a group's warps load the queries of a segment that it takes part in (as soon as they have
    seen the last scores of the one before it, where they had any, otherwise at its begin), see its scores, and in a tile that
    both groups share meet the other group at its end; the thread that issues a group's products waits for the queries, then
    issues the scores.  A segment is planned when the one PLANNED before it has been taken by all."""
    edges = {}

    def before(a, b):
        edges.setdefault(a, []).append(b)
    for h in (0, 1):
        at, product = ("begin", h), ("start", h)
        loads = []
        for i, (both, n) in enumerate(segments):
            count, takes = units_of(both, n, h), takes_part(both, n, h)
            taken = ("taken", h, i)
            before(product, taken)
            product = taken
            if i + PLANNED < len(segments):
                before(taken, ("planned", i + PLANNED))
            before(at, ("segment", h, i))
            before(("planned", i), ("segment", h, i))
            before(("planned", i), taken)
            at = ("segment", h, i)
            if takes:
                load = ("load", h, i)
                early = i and units_of(*segments[i - 1], h)      # under the last scores of the segment before
                before(("seen", h, i - 1) if early else at, load)
                before(("planned", i), load)
                loads.append(i)
                before(product, ("waited", h, i))
                before(load, ("waited", h, i))
                product = ("waited", h, i)
                before(load, ("ready", h, i))
                before(at, ("ready", h, i))
                at = ("ready", h, i)
            if count:
                before(product, ("issued", h, i))
                before(("issued", h, i), ("seen", h, i))
                before(at, ("seen", h, i))
                product, at = ("issued", h, i), ("seen", h, i)
            if not both:
                before(at, ("met", i))
                at = ("met", i)
        edges[("loads", h)] = loads

    def reaches(a, b):
        seen, todo = {a}, [a]
        while todo:
            x = todo.pop()
            if x == b:
                return True
            for y in edges.get(x, []):
                if y not in seen:
                    seen.add(y)
                    todo.append(y)
        return False
    return [(h, i, j) for h in (0, 1) for i, j in zip(edges[("loads", h)], edges[("loads", h)][1:]) if not reaches(("waited", h, i), ("load", h, j))]


def takes_part(units_of):
    return lambda both, n, h: units_of(both, n, h) > 0


@pytest.mark.parametrize("seed", range(60))
def test_queries_are_waited_for_before_the_next_ones_are_ready(units_of, seed):
    rs = np.random.RandomState(seed)
    segments = [(bool(rs.rand() < 0.4), int(rs.choice([1, 1, 1, 2, 3, 8]))) for _ in range(int(rs.randint(2, 14)))]
    assert unordered(segments, takes_part(units_of), units_of) == []


@pytest.mark.parametrize("segments", [[(True, 3), (False, 1), (False, 1)], [(False, 1)] * 6, [(True, 1), (False, 1), (True, 1), (False, 1), (False, 2)]])
def test_a_group_without_a_unit_takes_no_part(units_of, segments):
    assert unordered(segments, takes_part(units_of), units_of) == []
    # the model sees it where every group loads queries of every segment
    assert unordered(segments, lambda both, n, h: True, units_of) != []


def test_units_of_the_two_groups(units_of):
    for n in range(9):
        assert units_of(1, n, 0) == units_of(1, n, 1) == n
        assert [units_of(0, n, h) for h in (0, 1)] == [len(range(h, n, 2)) for h in (0, 1)]
