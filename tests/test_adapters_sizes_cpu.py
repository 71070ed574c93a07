"""Sizes that the library and its Python side share: which calls have many tokens, and the scratch they take."""
from __future__ import annotations

import pytest

from paper_2606_20855_gb300 import _abi, build, routing


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


@pytest.mark.parametrize("nrows,r,many", [(0, 16, False), (512, 16, False), (513, 16, True), (512, 1, False), (513, 1, True), (256, 17, False),
                                          (257, 17, True), (512, 0, False), (513, 0, True), (2, 4096, False), (3, 4096, True)])
def test_many_tokens(nrows, r, many):
    assert _abi.ws_adapters_many(nrows, r) is many and routing._adapters_many(nrows, r) is many


def test_scratch_comes_from_the_library(monkeypatch):
    """One place decides: another answer of the library's is what the calls go by."""
    for nnz, r in ((0, 8), (10, 9), (1000, 16)):
        assert routing._adapters_scratch(nnz, r) == _abi.ws_adapters_scratch(nnz, r)
    routing._adapters_scratch.cache_clear()
    routing._adapters_many.cache_clear()
    monkeypatch.setattr(_abi, "ws_adapters_scratch", lambda nnz, r: 12345)
    monkeypatch.setattr(_abi, "ws_adapters_many", lambda nrows, r: nrows > 7)
    assert routing._adapters_scratch(10, 9) == 12345 and routing._adapters_many(8, 1) and not routing._adapters_many(7, 999)
    routing._adapters_scratch.cache_clear()
    routing._adapters_many.cache_clear()
