"""The host side of the operators around a verification, without a GPU: how a commit's positions are shared out, what is refused."""
import ctypes as C
import glob
import os
import re

import pytest

from tests import servehost, serveplan, test_serve_plan

I, U, L, P = C.c_int, C.c_uint, C.c_int64, C.c_void_p


@pytest.fixture(scope="module")
def commit():
    return servehost.build("""
#include "commit_plan.hpp"
using namespace stand;
extern "C" {
int per_group(int row_words) { return commit_per_group(row_words); }
int64_t groups(int width, int per) { return commit_groups(width, per); }
int positions(int count, int width) { return commit_positions(count, width); }
int words(int n, unsigned j0, int per, int row_words) { return commit_words(n, j0, per, row_words); }
}""", dict(per_group=([I], I), groups=([I, I], L), positions=([I, I], I), words=([I, U, I, I], I)))


# kv heads * 16-byte words of a head's row: the smallest, ordinary ones, the largest that a cache may have
ROW_WORDS = [8, 16, 24, 64, 128, 512, 1024, 1040, 65536]


@pytest.mark.parametrize("row_words", ROW_WORDS)
def test_a_commit_copies_what_was_counted_and_nothing_else(commit, row_words):
    """At every position where a 32-bit product of positions and words could wrap, for every count."""
    per = commit.per_group(row_words)
    assert per >= 1 and (per == 1 or (per - 1) * row_words < 1024)
    wraps = [k * 2 ** 31 // row_words + e for k in (1, 2, 3) for e in (-per, -1, 0, 1, per)]
    for width in [1, 2, per, per + 1, 4099, 2 ** 24 + 5, 2 ** 30]:
        for count in [-2 ** 31, -2 ** 31 + 1, -1, 0, 1, per, 7, width - 1, width, width + 1, 2 ** 31 - 1]:
            n = commit.positions(count, width)
            assert n == min(max(count, 0), width)
            step = commit.groups(width, per) * per
            assert 1 <= commit.groups(width, per) < 2 ** 32 / 256        # threads of a launch's dimension
            last = (width - 1) // per * per
            for j0 in {0, per, last} | {x // per * per for x in wraps + [n - 1, n, n + per]}:
                if not 0 <= j0 <= last:
                    continue
                assert commit.words(n, j0, per, row_words) == min(max(n - j0, 0), per) * row_words, (width, count, j0)
            # a workgroup's next position: behind the last one it is past the end of every row, in 32 bits without a sign too
            assert n + step < 2 ** 32 and (step >= width or commit.groups(width, per) == (2 ** 32 - 1) // 256)


def test_scales_of_the_attention():
    """A scale's product with log2(e) is a number, however large the scale is."""
    L, c = serveplan.lib(), test_serve_plan.cache()

    def call(scale):
        rows = serveplan.TreeRows(d_q=4096, d_k=4096, d_v=4096, d_out=8192, q_heads=4, scale=scale)
        return L.attention(3, C.byref(c), 1, 64, 64, 9, 64, C.byref(rows), 256)

    for scale in (1e-45, 1e-38, 0.125, 1.0, 2.0 ** 127):
        assert call(scale) == 0, scale
    for scale in (0.0, -0.0, -1.0, 1.7015e38, 3.4e38, float("inf"), float("nan")):
        assert call(scale) == test_serve_plan.EINVAL, scale


@pytest.fixture(scope="module")
def checks():
    return servehost.build("""
#include "serve_checks.hpp"
using namespace stand;
extern "C" {
int sized(int64_t B, const stand_cache *c, int q_heads) { return check_attention_size(B, c, q_heads); }
int call(int64_t B, const stand_cache *c, const stand_tree_rows *r)
{
    const int32_t *x = (const int32_t *)64;
    return check_tree_attention(B, c, 0, x, x, 9, x, r, (const void *)256);
}
}""", dict(sized=([L, P, I], I), call=([L, P, P], I)))


def test_no_workspace_is_named_for_an_attention_that_is_refused(checks):
    """What the size of the workspace depends on is refused by both, by the same code."""
    far = dict(pages=2 ** 15 + 1, page_size=16)
    for B, q, kw in ((3, 4, {}), (4096, 4, {}), (4097, 4, {}), (65535, 4, {}), (3, 65534, {}), (3, 65535, {}), (3, 65536, {}), (3, 3, {}), (3, 0, {}), (3, -2, {}),
                     (3, 4, dict(far, page_stride=2 ** 20)), (3, 4, dict(far, page_stride=2 ** 20 - 128)), (3, 4, dict(page_size=4096, slot_stride=(1 << 48) - 8)),
                     (4097, 3, {}), *((3, 4, kw) for kw in test_serve_plan.BAD_CACHE)):
        c = test_serve_plan.cache(**kw)
        rows = serveplan.TreeRows(d_q=4096, d_k=4096, d_v=4096, d_out=8192, q_heads=q, scale=0.125)
        assert checks.sized(B, C.byref(c), q) == checks.call(B, C.byref(c), C.byref(rows)), (B, q, kw)


def test_words_of_a_row_are_aligned_like_its_elements():
    """What the shaped logits are read and written through promises no more than the accepted pointers keep (2 and 4 bytes)."""
    lib = servehost.build("""
#include "row_words.hpp"
using namespace stand;
template <int ES> static int sum(const char *row, int first)
{
    typedef typename RowWords<ES>::type Words;
    const Words w = *(const Words *)(row + first * ES);
    return (int)(w[0] + w[1] + w[2] + w[3]);
}
extern "C" {
int alignment(int es) { return es == 2 ? (int)alignof(RowWords<2>::type) : (int)alignof(RowWords<4>::type); }
int bytes(int es) { return es == 2 ? (int)sizeof(RowWords<2>::type) : (int)sizeof(RowWords<4>::type); }
int sum_at(int es, const void *row, int first) { return es == 2 ? sum<2>((const char *)row, first) : sum<4>((const char *)row, first); }
}""", dict(alignment=([I], I), bytes=([I], I), sum_at=([I, P, I], I)))
    row = (C.c_uint8 * 64)(*range(64))
    for es in (2, 4):
        assert lib.alignment(es) == es and lib.bytes(es) == 16
        for first in range(8):
            data = bytes(row)[first * es: first * es + 16]
            want = sum(int.from_bytes(data[4 * i: 4 * i + 4], "little") for i in range(4)) & 0xFFFFFFFF
            assert lib.sum_at(es, row, first) & 0xFFFFFFFF == want
    text = open(servehost.CSRC + "/shape_logits.hpp").read()
    rows = [line for line in text.splitlines() if "__builtin_nontemporal_" in line]
    assert rows and all("RowWords<" in line for line in rows)


def test_inline_assembly_writes_no_register_behind_the_compilers_back():
    """m0 and other registers by name are operands of the statements that need them, never written inside."""
    found = 0
    for path in glob.glob(os.path.join(servehost.CSRC, "*.h*")):
        for text in re.findall(r'asm volatile\(\s*"([^"]*)"', open(path).read()):
            found += 1
            for line in text.replace("\\t", "").split("\\n"):
                assert not re.match(r"\w+\s+(m0|vcc|exec|[sv]\d+|[sv]\[)", line.strip()), (path, line)
    assert found > 4


@pytest.mark.parametrize("kind", ["short", "any"])
def test_shares_of_heads_of_64_with_64_rows(kind):
    """The partition of the one form that tests/test_serve_plan.py leaves out: tiles of 64 rows, beginnings of eight units."""
    test_serve_plan.test_shares_cover_every_unit_once(kind, 64, 64, 8, 1, 1)
