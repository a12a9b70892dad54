"""atp_kv_extend as its seven launches (pools above 2^19 blocks, steps above
2^13 rows or tables above 2^17 entries; smaller ones take one workgroup, which
test_gpu_kv_ops.py covers): holes, shared blocks, every refusal, and good steps
behind refused ones on one workspace.  GPU, through the C ABI."""
import numpy as np
import pytest
import torch

from oracle import kvstep
from paper_2511_11617_amd import atp
from tests.test_gpu_kv_ops import check_extend, dev, random_step, stream

pytestmark = pytest.mark.gpu
POOL, ROWS, ENTRIES = (1 << 19) + 1, (1 << 13) + 1, (1 << 17) + 1  # the least of each that takes the launches


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()


def refusal(case, pool, rows):
    table, cached, fresh = [[0, 1, -1], [2, -1, -1], [4, 5, -1]], [5, 2, 8], [1, 2, 1]
    if case == "negative_cached":
        cached[1] = -1
    elif case == "negative_fresh":
        fresh[1] = -1
    elif case == "past_table":
        fresh[2] = 5
    elif case == "id_high":
        table[1][2] = pool
    elif case == "id_low":
        table[1][2] = -2
    elif case == "shared_written":
        table[2][0] = 1
    elif case == "twice_in_a_row":
        table[0] = [1, 1, -1]
    elif case == "overflow":
        cached[1], fresh[1] = 2 ** 31 - 1, 2 ** 31 - 1
    elif case == "past_rows":  # one row more than there are
        cols = -(-(rows + 9) // 4)
        table, cached, fresh = [[0, 1] + [-1] * cols, [2] + [-1] * (cols + 1), [4, 5] + [-1] * cols], [5, 2, 8], [1, 2, rows - 2]
        pool = max(pool, cols + 9)
    return table, cached, fresh, 4, pool, rows


REFUSALS = ["negative_cached", "negative_fresh", "past_table", "past_rows", "id_high", "id_low", "shared_written", "twice_in_a_row",
            "overflow"]


@pytest.mark.parametrize("by", ["pool", "rows"])
@pytest.mark.parametrize("case", REFUSALS)
def test_refusals(case, by):
    got = check_extend(*refusal(case, *((POOL, 5) if by == "pool" else (9, ROWS))))
    assert got[4] == [atp.EINVAL, 0, 0, 0]


def test_to_the_last_free_block_and_one_more():
    table = [[0, -1, -1], [3, -1, -1]]
    assert check_extend(table, [4, 2], [8, 6], 4, 5, ROWS)[4] == [0, 14, 3, 0]
    assert check_extend(table, [4, 2], [8, 7], 4, 5, ROWS)[4] == [atp.ECAPACITY, 0, 4, 3]
    assert check_extend(table, [4, 2], [8, 6], 4, 4, ROWS)[4] == [atp.ECAPACITY, 0, 3, 2]


def test_a_large_pool_to_its_last_block_and_one_more():
    """The last free id is the pool's last one; then one block too few."""
    cols = 1030
    table = np.full((512, cols), -1, np.int64)
    ids = np.random.default_rng(1).permutation(POOL - 1)
    table[:, :1024] = ids.reshape(512, 1024)  # all but the last id
    cached, fresh = [2 * 1024] * 512, [0] * 512
    fresh[300] = 2
    want = check_extend(table, cached, fresh, 2, POOL, 3)
    assert want[4] == [0, 2, 1, 0] and want[0][300, 1024] == POOL - 1
    fresh[7] = 1
    assert check_extend(table, cached, fresh, 2, POOL, 3)[4] == [atp.ECAPACITY, 0, 2, 1]


@pytest.mark.parametrize("by", ["pool", "rows", "entries"])
def test_holes_and_shared_prefixes(by):
    table, cached, fresh = random_step(9, 30, 20, 8, 1200, 50, holes=0.3)
    pool, rows = 1200, sum(fresh)
    if by == "pool":
        pool = POOL
    elif by == "rows":
        rows = ROWS
    else:  # a wider table
        table = np.concatenate([table, np.full((30, -(-ENTRIES // 30)), -1)], 1)
    assert check_extend(table, cached, fresh, 8, pool, rows)[4][0] == 0
    # a full block that several sequences name, and none writes
    table = np.full((3, 3 if by != "entries" else ENTRIES // 3 + 1), -1)
    table[:, 0] = 7
    table[0, 1], table[1, 1] = 0, 1
    assert check_extend(table, [6, 8, 4], [2, 1, 3], 4, max(9, pool * (by == "pool")), max(6, rows * (by == "rows")))[4][:3] == [0, 6, 2]


def test_no_sequence_and_no_token():
    assert check_extend(np.zeros((1, 2)) - 1, [0], [0], 4, POOL, 0)[4] == [0, 0, 0, POOL]
    assert check_extend(np.zeros((0, 2)), [], [], 4, POOL, 2)[4] == [0, 0, 0, POOL]


@pytest.mark.parametrize("by", ["pool", "rows"])
def test_good_steps_behind_refused_ones_on_one_workspace(by):
    """What a refused step leaves in the workspace changes nothing for the next."""
    pool, rows = (POOL, 60) if by == "pool" else (64, ROWS)
    good = ([[0, 1, -1], [2, -1, -1], [4, 5, -1]], [5, 2, 8], [4, 7, 1])
    full = ([list(range(20)), list(range(20, 40)), list(range(40, 59)) + [-1]], [0, 0, 76], [0, 0, 4])
    steps = [good, full]
    for case in REFUSALS:
        if case != "past_rows":
            steps += [refusal(case, pool, rows)[:3], good]
    n, most = 3, 20
    i32 = dict(dtype=torch.int32, device="cuda")
    table, new = torch.empty(n, most, **i32), torch.empty(n, most, **i32)
    cached, fresh, starts, status = torch.empty(n, **i32), torch.empty(n, **i32), torch.empty(n + 1, **i32), torch.empty(4, **i32)
    slots, pos = torch.empty(rows, dtype=torch.int64, device="cuda"), torch.empty(rows, **i32)
    cache = atp.KVCache(0, 0, 1, 4, 64, pool, (0, 0), (0, 0), 1)
    step = atp.KVStep(new.data_ptr(), n, most, cached.data_ptr(), fresh.data_ptr(), starts.data_ptr(), slots.data_ptr(), pos.data_ptr(),
                      rows, 0, 0, status.data_ptr())
    need = atp.kv_extend_workspace(cache, step)
    ws = torch.full((need,), 0xEE, dtype=torch.uint8, device="cuda")
    for t, c, f in steps:
        wide = np.full((n, most), -1, np.int32)
        wide[:, :len(t[0])] = t
        if f[2] == 5:
            f = [1, 2, 4 * most - 8 + 1]  # past the wider table too
        table.copy_(dev(wide, torch.int32))
        cached.copy_(dev(c, torch.int32))
        fresh.copy_(dev(f, torch.int32))
        atp.kv_extend(cache, step, table.data_ptr(), ws.data_ptr(), need, stream())
        torch.cuda.synchronize()
        want = kvstep.extend(wide, c, f, 4, pool, rows)
        got = (new.cpu().numpy(), starts.tolist(), slots.tolist(), pos.tolist(), status.tolist())
        assert np.array_equal(got[0], want[0]) and list(got[1:]) == list(want[1:]), (c, f, got[4], want[4])
