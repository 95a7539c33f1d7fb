"""The choice of continuations and the tables that follow it on the GPU at sizes where
their kernels go another way: rows of more than 64 table entries, tables on either side of
what one launch takes, rows of more than 64 chunks of the vocabulary."""
import numpy as np
import pytest
import torch

from paper_2609_39056_amd import binding as B
from test_beams_gpu import beams_state, check_reorder, check_select

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


# ------------------------------------------------------------------ tables
ONE_LAUNCH_WORDS = 36 << 10


def words(rows, max_pages, num_pages):
    """What a table takes of a workgroup's LDS: two words per page, three per row and its entries in runs of 64."""
    return 2 * num_pages + rows * (3 + 64 * -(-max_pages // 64))


def random_state(rng, rows, max_pages, num_pages, page=16, drop=0.3, full=0.5):
    """Rows that share pages as it happens, many of them with all their entries; some of the rows are dropped, so that
    pages come free from every part of a row."""
    table = rng.integers(0, num_pages, (rows, max_pages)).tolist()
    kv_len = [max_pages * page if rng.random() < full else int(rng.integers(0, max_pages * page + 1)) for _ in range(rows)]
    kept = [r for r in range(rows) if rng.random() >= drop] or [0]
    parent = [int(rng.choice(kept)) if rng.random() < 0.95 else -1 for _ in range(rows)]
    return table, kv_len, parent


@pytest.mark.parametrize("max_pages", [63, 64, 65, 128, 129, 142, 290])
@pytest.mark.parametrize("rows,num_pages", [(1, 3000), (5, 4000), (24, 9000)])
def test_reorder_long_rows(rows, max_pages, num_pages):
    # few rows, in one launch
    assert words(rows, max_pages, num_pages) <= ONE_LAUNCH_WORDS
    rng = np.random.default_rng([rows, max_pages])
    for trial in range(2):
        table, kv_len, parent = random_state(rng, rows, max_pages, num_pages)
        check_reorder(parent, kv_len, 16, num_pages, rng.permutation(num_pages).tolist(), num_pages // 2, table)
        check_reorder([-1] * rows, kv_len, 16, num_pages, rng.permutation(num_pages).tolist(), num_pages, table)


@pytest.mark.parametrize("rows,max_pages,num_pages", [(1000, 64, 40000), (1000, 65, 40000), (1000, 142, 60000), (1024, 290, 200000),
                                                      (40, 290, 30000), (8, 700, 40000)])
def test_reorder_long_rows_in_phases(rows, max_pages, num_pages):
    assert words(rows, max_pages, num_pages) > ONE_LAUNCH_WORDS
    rng = np.random.default_rng([rows, max_pages])
    table, kv_len, parent = random_state(rng, rows, max_pages, num_pages, drop=min(0.3, 30 / rows))
    want = check_reorder(parent, kv_len, 16, num_pages, rng.permutation(num_pages).tolist(), num_pages // 2, table)
    late = {p for s in set(range(rows)) - set(parent) for p in table[s][64:-(-kv_len[s] // 16)]}
    given = set(want[3]) | set(want[5][want[6]:num_pages // 2])
    assert max_pages <= 64 or late & given  # pages past entry 64 came free


@pytest.mark.parametrize("rows,max_pages,num_pages", [(64, 142, 12192), (64, 142, 12193), (550, 3, 7), (550, 3, 8), (551, 3, 7),
                                                      (189, 129, 0), (100, 290, 2282)])
def test_reorder_at_the_limit_of_one_launch(rows, max_pages, num_pages):
    num_pages = num_pages or (ONE_LAUNCH_WORDS - words(rows, max_pages, 0)) // 2
    assert abs(words(rows, max_pages, num_pages) - ONE_LAUNCH_WORDS) <= 128
    rng = np.random.default_rng([rows, max_pages, num_pages])
    table, kv_len, parent = random_state(rng, rows, max_pages, num_pages)
    check_reorder(parent, kv_len, 16, num_pages, rng.permutation(num_pages).tolist(), num_pages // 2, table)


@pytest.mark.parametrize("rows", [1023, 1024, 1025, 8191, 8192])
def test_reorder_many_short_rows(rows):
    rng = np.random.default_rng(rows)
    table, kv_len, parent = random_state(rng, rows, 2, 3 * rows, page=8, drop=0.1)
    check_reorder(parent, kv_len, 8, 3 * rows, rng.permutation(3 * rows).tolist(), rows, table)


@pytest.mark.parametrize("groups,beams,prompt,own", [(2, 4, 1600, 300), (16, 4, 2000, 260), (250, 4, 4000, 600)])
def test_reorder_long_prompts_after_a_choice(groups, beams, prompt, own):
    rng = np.random.default_rng([groups, prompt])
    table, kv_len, used, rest, num_pages = beams_state(rng, groups, beams, 16, prompt, own, 50)
    parent = [int(g * beams + rng.integers(0, beams)) for g in range(groups) for _ in range(beams)]
    check_reorder(parent, kv_len, 16, num_pages, used + rest, len(used), table)


# ------------------------------------------------------------------ choice
@pytest.mark.parametrize("width", [8, 64])
@pytest.mark.parametrize("kind", ["random", "equal", "near"])
def test_select_more_than_64_chunks(kind, width):
    """2^20 tokens are 128 chunks: a lane has two, and more keys than are ordered together.  Equal logits, and those that
    differ in the lower 16 bits only, leave every chunk's best in the list."""
    V = 1 << 20
    g = torch.Generator().manual_seed(width)
    if kind == "random":
        logits = torch.randn((2, V), generator=g) * 2.5
    elif kind == "equal":
        logits = torch.zeros((2, V))
    else:
        logits = 1.0 + torch.randint(0, 1 << 16, (2, V), generator=g) * 2.0 ** -23
    scores = torch.tensor([-1.0, -1.5])
    check_select(logits, scores, None, 0, 1, width)
    check_select(logits, scores, None, 0, 2, width)
    if kind == "equal":  # the best are in the last chunks of a lane's second half
        logits[:, V - 100:] = 1.0
        logits[:, 5] = 1.0
        check_select(logits, scores, None, 0, 2, width)


@pytest.mark.parametrize("V", [64 * 4096, 64 * 4096 + 1, 64 * 8192, 64 * 8192 + 1, 65 * 8192 + 3])
def test_select_around_64_chunks(V):
    logits = (torch.randint(0, 40, (4, V), generator=torch.Generator().manual_seed(V)) / 8).to(torch.bfloat16)
    check_select(logits, torch.tensor([0.0, -0.5, -30.0, -30.25]), None, 1, 2, 16)
