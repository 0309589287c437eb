"""What positions, the cache in 8 bits and the pages of a cache launch, without a GPU: calls of more threads than one launch holds, their slices,
forms, and what they ask for."""
import ctypes

import pytest

from test_history_launches_cpu import sums
from test_kernel_resources_cpu import scratch   # noqa: F401 (a fixture)
from test_launches_cpu import A, BF16, F32, launches, recorder   # noqa: F401 (a fixture)

SHAPE = 2


def attend(U, T, C, L, H, Hkv, D, dt, page=16):
    return lambda lib: lib.laser_cache8_attention_forward(A, H * D, A, A, A, A, A, A, A, U, T, C, 1 << 20, page, 8, 1 << 20, L, H, Hkv, D, 1.0, 1, dt,
                                                          A, A, A, 1 << 60, None)


def append(U, T, C, L, Hkv, D, dt, page=16, block=8):
    return lambda lib: lib.laser_cache8_append(A, Hkv * D, A, Hkv * D, A, A, A, A, A, A, A, U, T, C, 1 << 20, page, block, 1 << 20, L, Hkv, D, dt, None)


@pytest.mark.parametrize("dt,D,U,C,L,H,Hkv", [(BF16, 64, 9_000_000, 1, 500, 2, 2), (BF16, 128, 20_000_000, 1, 40, 1, 1), (F32, 64, 6_000_000, 3, 90, 6, 3),
                                             (BF16, 32, 5_000_000, 40, 90, 8, 4), (BF16, 64, 70_000, 1, 5000, 4, 2), (F32, 128, 300_000, 100, 300, 8, 8)])
def test_caches_of_many_users(recorder, dt, D, U, C, L, H, Hkv):
    seen = sums(launches(recorder, attend(U, U, C, L, H, Hkv, D, dt)))
    print({k[-60:]: v for k, v in seen.items()})
    (grids,) = seen.values()
    assert U * Hkv <= sum(grids) <= U * Hkv * (-(-C * H // Hkv // 32) + 3) + 32 * len(grids)


def test_too_many_workgroups_launch_nothing(recorder):
    recorder.launch_clear()
    assert attend((1 << 31) - 1, 5, 1, 16, 2, 2, 16, BF16)(recorder) == SHAPE
    assert append(1, 1 << 22, 1 << 22, 1 << 22, 64, 16, BF16)(recorder) == SHAPE
    assert recorder.launch_count() == 0


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("U,C,Hkv,block", [((1 << 31) - 1, 1, 1, 8), (70_000, 1, 2, 16), (400, 100_000, 8, 8), (3, 1, 1024, 16)])
def test_appends_cover_every_user(recorder, U, C, Hkv, block, dt):
    T = min(C, 100_000) if U < 1000 else 5
    records = launches(recorder, append(U, T, C, 100_000, Hkv, 16, dt, block=block))
    blocks = (C + 2 * block - 2) // block
    users = min(65535, ((1 << 32) - 1) // 256 // (blocks * Hkv * 2))      # of a launch, the third side of its grid
    assert len(records) == -(-U // users) and all(r.grid == blocks and r.block == 256 for r in records)


#       U  Hkv H    L   C   waves  runs
FORMS = [(1, 2, 16, 65000, 1, 8, 127), (8, 2, 8, 20000, 1, 8, 20), (40, 2, 8, 3000, 1, 8, 3), (128, 2, 8, 4096, 1, 4, 4), (256, 2, 8, 2000, 4, 4, 1),
         (5, 2, 4, 777, 1, 8, 1), (200, 1, 4, 5000, 1, 4, 5), (600, 1, 4, 100000, 2, 4, 1), (100, 2, 8, 3000, 1, 8, 1), (65, 2, 8, 3201, 8, 4, 4)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("U,Hkv,H,L,C,waves,runs", FORMS)
def test_forms_of_few_rows(recorder, U, Hkv, H, L, C, waves, runs, dt):
    """Runs and waves by the rules beside cache8_runs_of; the work buffer holds what the runs leave; a join follows where there are several."""
    for D in (32, 64, 128):
        records = launches(recorder, attend(U, U * C, C, L, H, Hkv, D, dt))
        first = records[0]
        assert "cache8_few_kernel" in first.kernel.decode() and first.block == 64 * waves and first.grid == U * Hkv * runs
        assert len(records) == (2 if runs > 1 else 1) and all("join" in r.kernel.decode() for r in records[1:])
        need = recorder.laser_cache8_attention_work_bytes(U, U * C, C, L, H, Hkv, D, dt)
        assert need == (runs * U * C * H * (D + 1) * 4 if runs > 1 else 16)


@pytest.mark.parametrize("U,Hkv,H,L,C,D,runs", [(16, 2, 8, 10000, 512, 128, 3), (64, 2, 8, 4096, 256, 64, 2), (65, 2, 8, 4096, 256, 64, 2), (1, 2, 8, 30000, 100, 128, (59, 118)),
                                                (1, 2, 8, 1000, 100, 64, 4), (200, 1, 8, 100, 500, 32, 1), (50, 2, 8, 1500, 1000, 128, 1), (256, 2, 8, 1000, 32, 128, 1), (255, 2, 8, 1000, 32, 128, 4), (256, 2, 8, 1025, 32, 128, 4), (1, 1, 1, 5000, 128, 128, (10, 20)), (32, 2, 8, 4096, 16, 128, (8, 16)),
                                                (3, 1, 1, 384, 33, 64, 1), (2, 1, 1, 385, 65, 32, 2)])
def test_forms_of_many_rows(recorder, U, Hkv, H, L, C, D, runs):
    """Runs by the rules beside cache8_runs_of. Up to 64 users a workgroup for each tile and run; more in the dealt order, a multiple of eight;
    so do very many workgroups, of rows enough."""
    for dt, runs in zip((BF16, F32), runs if isinstance(runs, tuple) else (runs, runs)):
        records = launches(recorder, attend(U, U * C, C, L, H, Hkv, D, dt))
        rows = C * (H // Hkv)
        split = 2 if rows <= 64 or U * Hkv * -(-rows // 128) * runs <= 256 else 1      # (waves that have the same rows)
        workgroups = U * Hkv * -(-rows * split // 128) * runs
        assert "cache8_tile_kernel" in records[0].kernel.decode() and records[0].block == 256
        assert f"ELi{split}E{'f' if dt == F32 else 't'}E" in records[0].kernel.decode()
        assert records[0].grid == workgroups if U <= 64 and workgroups <= 2560 else workgroups <= records[0].grid < workgroups * 1.1 + 64
        assert len(records) == (2 if runs > 1 else 1) and all("join" in r.kernel.decode() for r in records[1:])
        assert recorder.laser_cache8_attention_work_bytes(U, U * C, C, L, H, Hkv, D, dt) == (runs * U * C * H * (D + 1) * 4 if runs > 1 else 16)


@pytest.mark.parametrize("U,H,L,C,D,kernel", [(1, 16, 65000, 1, 128, "cache8_join_kernel"), (1, 8, 8000, 1, 128, "cache_join_few_kernel"),
                                              (8, 8, 20000, 1, 128, "cache8_join_kernel"), (1, 8, 30000, 100, 128, "cache_join_kernel")])
def test_joins(recorder, U, H, L, C, D, kernel):
    """More than 16 parts of few rows, of many, and few parts."""
    for dt in (F32, BF16):
        records = launches(recorder, attend(U, U * C, C, L, H, 2, D, dt))
        assert len(records) == 2 and kernel in records[1].kernel.decode()


def test_positions_of_many_rows(recorder):
    T = (1 << 31) // 8 - 1
    for D, layout in ((8, 0), (128, 1)):
        records = launches(recorder, lambda lib: lib.laser_rotary_forward(A, 8 * D, None, 0, A, A, T, 8, 0, D, D, layout, 1.0, BF16, A, 8 * D, None, 0, None))
        tokens = 16 if D == 8 else 5      # (a piece or two for each of 256 threads; 16 at most)
        assert sum(r.grid for r in records) == -(-T // tokens) and all(r.grid * r.block < 1 << 32 for r in records)


@pytest.mark.parametrize("n", [1, 16, 17, 1000])
def test_parts_of_a_page_by_sixteen(recorder, n):
    parts = (ctypes.c_void_p * n)(*[A] * n), (ctypes.c_int64 * n)(*[4096] * n)
    records = launches(recorder, lambda lib: lib.laser_pages_copy(*parts, n, A, A, 3, 100, None))
    assert len(records) == -(-n // 16) and sum(r.grid for r in records) == sum(-(-3 * 256 * min(16, n - i) // 256) for i in range(0, n, 16))
    fork = launches(recorder, lambda lib: lib.laser_pages_fork(*parts, n, A, A, A, A, 2, 3, 8, 16, 4, 4, A, A, A, A, 1 << 30, None))
    assert len(fork) == (1 if n == 1 else 1 + -(-n // 16))      # (a small one is one workgroup's, plan and all)


@pytest.mark.parametrize("P,plans", [(1, 1), (4096, 1), (4097, 1), (16384, 1), (16385, 2), (1 << 26, 2)])
def test_compaction_without_parts(recorder, P, plans):
    """Tables and counts alone: the plan and one launch, for pools of any size."""
    records = launches(recorder, lambda lib: lib.laser_pages_compact(None, None, 0, A, A, A, 2, P, 16, 4, A, A, A, A, 1 << 40, None))
    assert len(records) == plans + 1 and all(r.grid * r.block < 1 << 32 for r in records)


@pytest.mark.parametrize("P,counts", [(32768, 0), (32769, 1), (1 << 26, 1)])
def test_taking_pages_of_a_large_pool(recorder, P, counts):
    """Chunks that are full are counted ahead, and a fork is then never one workgroup's."""
    grow = launches(recorder, lambda lib: lib.laser_pages_grow(A, A, A, A, 2, P, 16, 4, A, A, 1 << 40, None))
    assert len(grow) == 1 + counts and all(r.grid * r.block < 1 << 32 for r in grow)
    part = (ctypes.c_void_p * 1)(A), (ctypes.c_int64 * 1)(4096)
    fork = launches(recorder, lambda lib: lib.laser_pages_fork(*part, 1, A, A, A, A, 2, 3, P, 16, 4, 4, A, A, A, A, 1 << 40, None))
    assert len(fork) == (1 if not counts else 3)


def test_no_kernel_uses_scratch(scratch):
    kernels = {k: n for k, n in scratch.items() if "5laser" in k and any(name in k for name in (
        "cache8_", "rotary_", "fork_", "grow_kernel", "free_kernel", "used_kernel", "compact_", "copy_kernel"))}
    assert len(kernels) >= 30 and not {k: n for k, n in kernels.items() if n}
