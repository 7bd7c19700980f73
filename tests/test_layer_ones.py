"""Dimensions of one element: their strides mean nothing, and the binding of the layer's blocks
does not look at them. No GPU is used."""
from __future__ import annotations

import pytest
import torch

import paper_2607_08973_amd as S
from test_layer_refusals import D, HQ, PAGE, PAGES, T, i32, recorder, z  # noqa: F401


def caches(kind):
    """Of one head, pages [PAGES][PAGE][1][D]: alike in memory, whatever the strides of the head
    say."""
    k = z(PAGES, PAGE, 1, D)
    return k, {"heads first": z(PAGES, 1, PAGE, D).transpose(1, 2),
               "strided": z(PAGES, PAGE, D).as_strided((PAGES, PAGE, 1, D), (PAGE * D, D, 12345, 1)),
               }[kind]


@pytest.mark.parametrize("kind", ["heads first", "strided"])
def test_caches_of_one_head(recorder, kind):  # noqa: F811
    k, v = caches(kind)
    assert k.stride() != v.stride()
    x = z(T, HQ + 2, D)
    for a, b in ((k, v), (v, k)):
        S.sifar_cache_append(x[:, HQ:HQ + 1], x[:, HQ + 1:], i32(T), i32(T, 3), a, b)
        S.sifar_paged_attention(z(T, HQ, D), a, b, i32(T, 1), i32(T), z(T, HQ, D))
    for c in recorder.calls:
        assert (c.page_stride, c.slot_stride) == (PAGE * D, D)


def test_a_cache_of_one_page_and_of_pages_of_one_slot(recorder):  # noqa: F811
    for shape in ((1, PAGE, 2, D), (PAGES, 1, 2, D)):
        k = z(*shape)
        at = list(k.stride())
        at[shape.index(1)] = 8
        v = z(*shape).as_strided(shape, at)
        S.sifar_paged_attention(z(T, HQ, D), k, v, i32(T, 1), i32(T), z(T, HQ, D))
    assert len(recorder.calls) == 2


def test_a_table_of_one_column(recorder):  # noqa: F811
    pages = torch.arange(T, dtype=torch.int32).view(1, T).t()  # [T][1], strides (1, T)
    assert pages.stride() == (1, T)
    k = z(PAGES, PAGE, 2, D)
    S.sifar_paged_attention(z(T, HQ, D), k, k.clone(), pages, i32(T), z(T, HQ, D))
    wide = i32(T, 5)[:, 2:3]
    S.sifar_paged_attention(z(T, HQ, D), k, k.clone(), wide, i32(T), z(T, HQ, D))
    assert [c.pages_stride for c in recorder.calls] == [1, 5]


def test_strides_that_mean_something_are_looked_at(recorder):  # noqa: F811
    k = z(PAGES, PAGE, 2, D)
    for v in (z(PAGES, 2, PAGE, D).transpose(1, 2), z(2 * PAGES, PAGE, 2, D)[::2]):
        with pytest.raises(S.SifarError):
            S.sifar_paged_attention(z(T, HQ, D), k, v, i32(T, 1), i32(T), z(T, HQ, D))
    with pytest.raises(S.SifarError):
        S.sifar_paged_attention(z(T, HQ, D), k, k.clone(), i32(2, T).t(), i32(T), z(T, HQ, D))
    assert not recorder.calls
