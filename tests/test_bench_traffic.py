"""The digest that ties the committed traffic figures to the step kernel's sources: it follows
these, and only these, and the figures are those of the present ones."""
import os
import shutil

import pytest

import bench


@pytest.fixture
def sources(tmp_path, monkeypatch):
    """A copy of the sources that the digest is taken over."""
    dirs = tuple(str(tmp_path / str(i)) for i in range(len(bench.SOURCE_DIRS)))
    for src, dst in zip(bench.SOURCE_DIRS, dirs):
        shutil.copytree(src, dst)
    monkeypatch.setattr(bench, "SOURCE_DIRS", dirs)
    return {name: os.path.join(d, name) for d in dirs for name in os.listdir(d)}


def _edit(path, at=None):
    """Adds a comment behind `at`, or at the end."""
    text = open(path).read()
    cut = len(text) if at is None else text.index(at) + len(at)
    open(path, "w").write(text[:cut] + "\n// another line\n" + text[cut:])


def test_the_digest_leaves_the_serving_calls_out(sources):
    before = bench.source_digest()
    for name in (*bench.DIGEST_SKIP, "kvec_bind.cpp"):
        _edit(sources[name])
    _edit(sources["kvec.h"])
    _edit(sources["kvec.h"], "kvec_prefill_workspace_size(")
    assert bench.source_digest() == before


@pytest.mark.parametrize("name,at", [("kvec.h", "kvec_select_cover("), ("kvec_pipeline.hip", None), ("kvec_score_dev.h", None),
                                     ("kvec_select_dev.h", None), ("kvec_step_inst.hip", None), ("kvec_internal.h", None)])
def test_the_digest_follows_the_step_kernel(sources, name, at):
    before = bench.source_digest()
    _edit(sources[name], at)
    assert bench.source_digest() != before


@pytest.mark.parametrize("workload", ["llama8b-32k", "llama8b-32k-lse"])
def test_the_committed_figures_are_those_of_the_present_kernels(workload):
    got = bench.measured_traffic(workload)
    assert isinstance(got, int) and got > 56_574_333  # the algorithmic bytes of a launch
