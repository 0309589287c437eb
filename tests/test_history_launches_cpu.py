"""What attention among a history's items launches, without a GPU: calls of more threads than one launch holds, their slices, and forms."""
import pytest

from test_history_f32_forms_gpu import CACHED, PACKED as F32_PACKED, lengths
from test_launches_cpu import A, BF16, F32, launches, recorder   # noqa: F401 (a fixture)

SHAPE = 2
THREADS = 1 << 32     # a launch holds fewer


def forward(N, T, L, H, Hkv, D, dt):
    return lambda lib: lib.laser_history_attention_forward(A, H * D, A, Hkv * D, A, Hkv * D, A, N, T, L, H, Hkv, D, 1.0, dt, A, A, None)


def backward(N, T, L, H, Hkv, D, dt):
    return lambda lib: lib.laser_history_attention_backward(A, H * D, A, Hkv * D, A, Hkv * D, A, A, A, A, N, T, L, H, Hkv, D, 1.0, dt, A, H * D,
                                                            A, Hkv * D, A, Hkv * D, A, 1 << 50, None)


def attend(U, T, C, L, H, Hkv, D, dt):
    return lambda lib: lib.laser_cache_attention_forward(A, H * D, A, A, A, A, A, U, T, C, 1 << 20, 16, 1 << 20, L, H, Hkv, D, 1.0, 1, dt, A, A, A,
                                                         1 << 50, None)


def sums(records):
    """{kernel: workgroups of all its launches}; every launch holds fewer than 2^32 threads."""
    out = {}
    for r in records:
        assert r.grid > 0 and r.grid * r.block < THREADS, (r.kernel, r.grid, r.block)
        out.setdefault(r.kernel.decode(), []).append(r.grid)
    return out


#              N        T          L      H Hkv  D
PACKED = [(100_000, 10_000_000, 8000, 4, 4, 32), (100_000, 10_000_000, 8000, 4, 4, 128), (3_000_000, 4_000_000, 700, 4, 2, 64),
          (9_000_000, 9_000_000, 20, 2, 2, 64), (2, 100, 50, 4, 2, 64), (300, 100_000, 5000, 8, 2, 128)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("N,T,L,H,Hkv,D", PACKED)
def test_packed_batches_with_a_long_outlier(recorder, N, T, L, H, Hkv, D, dt):
    """Grids grow with N * L_max, whatever T is: they go out in slices that hold whole sequences, and cover all of them."""
    for call, kernels in ((forward, 1), (backward, 2)):
        seen = sums(launches(recorder, call(N, T, L, H, Hkv, D, dt)))
        print(call.__name__, {k[-60:]: v for k, v in seen.items()})
        assert len(seen) == kernels
        for grids in seen.values():
            # tiles of 32 to 128 rows or items, whole eights of workgroups (of runs of four tiles) in each launch
            least, most = N * Hkv * -(-L // 128), N * Hkv * (-(-L * H // Hkv // 32) + 3)
            assert least <= sum(grids) <= most + 32 * len(grids)
            assert all(g % 8 == 0 for g in grids) and max(grids) == grids[0]


def test_a_call_of_too_many_workgroups_launches_nothing(recorder):
    """More than 2^31 - 1 workgroups, counted in the tiles of the form that the call has: refused as a whole, both ways."""
    for call in (forward, backward):
        for dt in (F32, BF16):
            recorder.launch_clear()
            assert call(1 << 30, 1 << 20, 1 << 20, 64, 64, 64, dt)(recorder) == SHAPE and recorder.launch_count() == 0
    # what the forward pass takes the backward pass takes: 2^29 workgroups of 128 rows, 2^31 of 32
    for call in (forward, backward):
        recorder.launch_clear()
        assert call(1 << 20, 1 << 20, 1 << 16, 1, 1, 64, BF16)(recorder) == 0, call.__name__


@pytest.mark.parametrize("dt,D,U,C,L,H,Hkv", [(BF16, 64, 9_000_000, 1, 500, 2, 2), (BF16, 128, 20_000_000, 1, 40, 1, 1), (F32, 64, 6_000_000, 3, 90, 6, 3),
                                             (BF16, 32, 5_000_000, 40, 90, 8, 4), (BF16, 64, 70_000, 1, 5000, 4, 2)])
def test_caches_of_many_users(recorder, dt, D, U, C, L, H, Hkv):
    seen = sums(launches(recorder, attend(U, U, C, L, H, Hkv, D, dt)))
    print({k[-60:]: v for k, v in seen.items()})
    (grids,) = seen.values()
    assert U * Hkv <= sum(grids) <= U * Hkv * (-(-C * H // Hkv // 32) + 3) + 32 * len(grids)


@pytest.mark.parametrize("U,budget", [(4_300_000, 1), (1 << 22, 500), ((1 << 22) - 1, 3), (70_000, 20), (3, 1000)])
def test_eviction_of_many_users(recorder, U, budget):
    """The selection, a workgroup of 1024 threads a user, covers every user in launches that hold it, all of them ahead of the moves."""
    records = launches(recorder, lambda lib: lib.laser_cache_evict(A, A, A, A, A, A, U, 1 << 20, 16, 64, 64, 1000, budget, 0, 2, 64, BF16, A, A, None))
    names = [r.kernel.decode() for r in records]
    seen = sums(records)
    select, = (grids for name, grids in seen.items() if "cache_select_kernel" in name)
    assert sum(select) == U and all("cache_select_kernel" in n for n in names[:len(select)])
    assert all("cache_move_kernel" in n for n in names[len(select):]) and len(names) - len(select) == -(-U // 65535)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_as_many_users_as_an_int_counts(recorder, dt):
    """Slices of 65535 users up to the last user that there can be."""
    U, D = (1 << 31) - 1, 8
    slices = -(-U // 65535)
    append = lambda lib: lib.laser_cache_append(A, D, A, D, A, A, A, A, A, U, 5, 1, 9, 16, 1, 16, 1, D, dt, A, None)
    weights = lambda lib: lib.laser_cache_weights(A, D, A, A, A, A, A, U, 5, 1, 9, 16, 1, 16, 1, 1, D, 1.0, 1, 1, dt, A, None)
    evict = lambda lib: lib.laser_cache_evict(A, A, A, A, A, A, U, 9, 16, 1, 1, 16, 1, 0, 1, D, dt, A, A, None)
    assert len(launches(recorder, append)) == slices and len(launches(recorder, weights)) == slices
    grids = sums(launches(recorder, evict))
    assert {k for k, v in grids.items() if len(v) == slices and "cache_move_kernel" in k} and U in [sum(v) for v in grids.values()]
    grids, = sums(launches(recorder, attend(U, 5, 1, 16, 1, 1, D, dt))).values()
    assert U <= sum(grids) <= U + 8 * len(grids)
    for call in (forward, backward):
        for grids in sums(launches(recorder, call(U - 7, 5, 16, 1, 1, D, dt))).values():
            assert U - 7 <= sum(grids) <= U - 7 + 8 * len(grids)


@pytest.mark.parametrize("N,L,H,Hkv,D,split,items", F32_PACKED)
def test_forms_of_packed_calls_in_single_precision(recorder, N, L, H, Hkv, D, split, items):
    T = sum(lengths(N, L)) + 5
    first, dq, dkv = (r.kernel.decode() for call in (forward, backward) for r in launches(recorder, call(N, T, L, H, Hkv, D, F32)))
    print(first, dq, dkv)
    assert "history_f32_kernelILi" in first and f"Lb0ELb{int(split)}EE" in first
    assert "history_dq_f32" in dq and f"ELb{int(split)}EE" in dq and "history_dkv_f32" in dkv and f"ELb{int(items)}EE" in dkv


@pytest.mark.parametrize("U,C,L,H,Hkv,D,page,split", CACHED)
def test_forms_of_cached_calls_in_single_precision(recorder, U, C, L, H, Hkv, D, page, split):
    T = sum(C if i % 3 else (i * 11) % (C + 1) for i in range(U)) + 3
    for causal in (0, 1):
        first = launches(recorder, lambda lib: lib.laser_cache_attention_forward(A, H * D, A, A, A, A, A, U, T, C, 1 << 20, page, 1 << 20, L, H, Hkv, D, 1.0,
                                                                                causal, F32, A, A, A, 1 << 50, None))[0]
        print(first.kernel)
        assert f"Lb1ELb{int(split)}EE" in first.kernel.decode()
