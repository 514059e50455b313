"""eg_mla_page_plan and eg_mla_page_release against the plain rules, one sequence after the other: equal to the last bit."""
import numpy as np
import pytest
import torch

import server_oracle as S
from paper_2509_16686_amd import binding as B
from parity import say

pytestmark = pytest.mark.gpu
I32 = torch.int32


def dev(x):
    return torch.tensor(np.asarray(x), dtype=I32, device="cuda")


def run_plan(page, cached, new, table, free, count, max_tokens, base=None, stream=None):
    b = len(cached)
    out = {k: torch.full((n,), -7, dtype=I32, device="cuda")
           for k, n in dict(lens=b, cu=b + 1, positions=max_tokens, slots=max_tokens, count=1).items()}
    t = dev(table).reshape(b, -1).contiguous()
    B.page_plan(page, dev(cached), dev(new), t, dev(free), dev([count]), out["lens"], out["cu"], out["positions"],
                out["slots"], out["count"], position_base=None if base is None else dev(base), stream=stream)
    torch.cuda.synchronize()
    return [t.cpu().numpy()] + [out[k].cpu().numpy() for k in ("lens", "cu", "positions", "slots")] + [int(out["count"])]


def check_plan(page, cached, new, table, free, count, max_tokens, base=None):
    got = run_plan(page, cached, new, table, free, count, max_tokens, base)
    i64 = [np.asarray(x, dtype=np.int64) for x in (cached, new, table, free)]
    want = S.page_plan(page, i64[0], i64[1], None if base is None else np.asarray(base), i64[2], i64[3], count, max_tokens)
    for name, g, w in zip(("table", "lens", "cu", "positions", "slots", "count"), got, want):
        assert np.array_equal(g, w), (name, g, w)
    return got


def random_step(seed, b, page, top_len, top_new, spare):
    r = np.random.default_rng(seed)
    cached, new = r.integers(0, top_len + 1, b), r.integers(0, top_new + 1, b)
    width = S.ceil_div(top_len + top_new, page)
    per = -(-cached // page)
    need = int((-(-(cached + new) // page) - per).sum())
    pages = r.permutation(int(per.sum()) + need + 40)
    table, at = np.full((b, width), -1, dtype=np.int64), 0
    for i, n in enumerate(per):
        table[i, :n] = pages[at:at + n]
        at += n
    return cached, new, table, pages[at:], need + spare, int(new.sum())


@pytest.mark.parametrize("b", [1, 2, 63, 64, 65, 255, 257, 1000, 4096])
@pytest.mark.parametrize("page", [1, 24, 64])
def test_plan_matches_the_rules(gpu, b, page):
    say(f"page_plan b={b} page={page}")
    cached, new, table, free, count, total = random_step(b, b, page, 200 if b < 1000 else 40, 90 if b < 1000 else 9, 3)
    check_plan(page, cached, new, table, free, min(count, len(free)), total + 11, base=np.arange(b) * 3)


@pytest.mark.parametrize("lack", [1, 5, 10 ** 6])
def test_too_few_pages_serve_the_first_sequences_and_those_that_need_none(gpu, lack):
    say(f"page_plan lack={lack}")
    cached, new, table, free, count, total = random_step(7, 130, 16, 100, 20, 0)
    got = check_plan(16, cached, new, table, free, max(count - lack, 0), total)
    assert (got[1] == cached + new).sum() < 130 and got[5] >= 0


def test_long_calls_over_many_work_groups(gpu):
    cached, new, table, free, count, total = random_step(9, 37, 64, 3000, 9000, 0)
    say(f"page_plan tokens={total}")
    check_plan(64, cached, new, table, free, count, total + 3)


@pytest.mark.parametrize("cut", [0, 1, 40, 100])
def test_tokens_past_the_arrays_are_not_taken_in(gpu, cut):
    say(f"page_plan cut={cut}")
    cached, new, table, free, count, total = random_step(3, 20, 8, 50, 30, 5)
    check_plan(8, cached, new, table, free, min(count, len(free)), max(total - cut, 0))


def test_values_out_of_range_are_made_safe(gpu):
    say("page_plan out of range")
    big = 2 ** 31 - 1
    # lengths below zero and above the row, a row outgrown, sums past 32 bits, page numbers that have no slots
    check_plan(16, [-5, 1000, 10, 0, 3, 0], [4, 1, 60, big, big, 3], np.array([[5, 6, 7, 8]] * 6), [9, -1, big, 4, 2], 5, 50)
    check_plan(16, [10, 20], [3, 20], np.array([[-1, 0, 0, 0], [3, big, 0, 0]]), [1, 2], 2, 40)
    # a count outside the stack
    check_plan(16, [0, 0], [3, 20], np.full((2, 4), -1), [1, 2], -3, 40)
    check_plan(16, [0, 0], [3, 20], np.full((2, 4), -1), [1, 2], 99, 40)
    # no free pages at all, no new tokens, no room in the token arrays
    check_plan(16, [3, 0], [3, 20], np.full((2, 4), 1), [], 0, 40)
    check_plan(16, [3, 0], [0, 0], np.full((2, 4), 1), [8], 1, 0)


@pytest.mark.parametrize("b,every", [(1, 1), (50, 3), (300, 2), (4096, 5)])
def test_release_matches_the_rules(gpu, b, every):
    say(f"page_release b={b}")
    r = np.random.default_rng(b)
    page, width = 16, 7
    lens, table = r.integers(-3, 130, b), r.permutation(b * width).reshape(b, width)
    ended = (np.arange(b) % every == 0).astype(np.int64) * r.integers(1, 5, b)
    whole = S.page_release(page, lens, ended, table, np.full(b * width + 9, -1), 4)
    for room in (b * width + 9, 4 + (whole[2] - 4) // 2, 4, 2):  # all come back, some are dropped, no room
        free = np.full(room, -1)
        want = S.page_release(page, lens, ended, table, free, 4)
        f, out, count = dev(free), torch.full((b,), -7, dtype=I32, device="cuda"), dev([-7])
        B.page_release(page, dev(lens), dev(ended), dev(table), f, dev([4]), out, count)
        torch.cuda.synchronize()
        assert np.array_equal(f.cpu().numpy(), want[0]) and np.array_equal(out.cpu().numpy(), want[1])
        assert int(count) == want[2]


def test_plan_on_another_stream_and_replayed(gpu):
    say("page_plan captured")
    cached, new, table, free, count, total = random_step(21, 40, 16, 100, 30, 0)
    s = torch.cuda.Stream()
    args = [dev(cached), dev(new), dev(table).reshape(40, -1).contiguous(), dev(free), dev([count])]
    out = [torch.empty(n, dtype=I32, device="cuda") for n in (40, 41, total, total, 1)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.page_plan(16, *args, *out)
    for step in range(3):  # other lengths in the same arrays
        c = np.asarray(cached) // (step + 1)
        args[0].copy_(dev(c))
        args[2].copy_(dev(table).reshape(40, -1))
        g.replay()
        torch.cuda.synchronize()
        want = S.page_plan(16, np.asarray(c), np.asarray(new), None, np.asarray(table), np.asarray(free), count, total)
        for got, w in zip([args[2]] + out, want):
            assert np.array_equal(got.cpu().numpy().reshape(-1), np.asarray(w).reshape(-1))
