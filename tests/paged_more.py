"""Further cases of the paged cache's calls: those that reach the kernels' instances and plans that the shorter ones do not."""
import paged_util as u

A, N = u.A, u.N
MANY = [
    u.case(dtype="f32", n=300, heads=(1, 1), lengths=((350,),), page=16),                                        # f32 rows of 512 bytes: four waves
    u.case(dtype="f32", n=130, heads=(4, 2), lengths=((1300, 200),), by_head=True, page=64),                     # ... long enough for chunks
    u.case(dtype="f32", n=257, heads=(32, 32), lengths=tuple((257 + 40 * b,) * 32 for b in range(4)), page=32),  # eight waves
    u.case(dtype="f32", d=64, n=257, heads=(32, 32), lengths=((257,) * 32, (300,) * 32, (20,) * 32, (257,) * 32),
           counts=((257,) * 32, (257,) * 32, (257,) * 32, (3,) * 32), page=16),                                  # eight waves; rows that are not there
    u.case(n=257, heads=(32, 32), lengths=tuple((257 + 100 * b,) * 32 for b in range(4)), page=16),              # bf16, eight waves, rows of 256 bytes
    u.case(dtype="f32", d=64, n=100, heads=(8, 1), lengths=((700,), (90,)), page=16, pool_token_major=True),     # f32, four waves, chunks
    u.case(dtype="f32", d=64, n=1, heads=(4, 1), lengths=((600,),), page=16),                                    # f32, chunks joined in the same launch
    u.case(dtype="f32", n=2, heads=(3, 1), lengths=((500,),), page=8),
    u.case(dtype="f32", n=3, heads=(12, 4), lengths=((300, 40, 1, 3),) * 2, by_head=True, page=8),                 # f32, one column tile, short
]

# rows: several tokens of a workgroup, the last of them not all there; several KV heads, the last group of them shorter; more of both than go abreast
_odd = lambda n, Hkv: ((n,) * Hkv, tuple(max(n - 1 - 977 * g, 3) for g in range(Hkv)))  # noqa: E731
ROWS = [
    u.case(n=8300, heads=(6, 3), lengths=_odd(8300, 3)[1:], counts=_odd(8300, 3)[1:], norm=True, rot_dim=128, by_head=True, page=64),
    u.case(d=64, n=2500, heads=(10, 5), lengths=((2600,) * 5,), norm=True, rot_dim=48, pairing=N, page=16),
    u.case(n=300, heads=(40, 40), lengths=((300,) * 40,), counts=((300,) * 37 + (299, 100, 0),), rot_dim=64, page=32),
    u.case(dtype="f32", n=2101, heads=(40, 20), lengths=((2101,) * 20,), norm=True, rot_dim=16, pairing=N, page=8, token_major=False),
    u.case(dtype="f32", d=64, n=1050, heads=(9, 9), lengths=_odd(1050, 9) * 4, counts=_odd(1050, 9) * 4, rot_dim=64, by_head=True, page=128),
    u.case(n=4111, heads=(2, 2), lengths=((5000, 4111),), counts=((4111, 4000),), by_head=True, page=16, pool_token_major=True),     # copies
    u.case(dtype="f32", d=64, n=4099, heads=(33, 33), lengths=((4099,) * 33,), page=256),                                            # copies
    u.case(dtype="f32", n=5, heads=(6, 2), lengths=((5, 9), (70, 70)), norm=True, rot_dim=128, page=4),
    u.case(dtype="f32", d=64, n=7, heads=(4, 4), lengths=((7, 9, 30, 31),), counts=((7, 1, 0, 5),), norm=True, rot_dim=24, pairing=N, by_head=True, page=2),
    u.case(d=64, n=21, heads=(3, 3), lengths=((21, 40, 300),), by_head=True, page=16),                                               # copies
    u.case(n=2051, heads=(8, 2), lengths=((2100, 2100),), norm=True, rot_dim=128, pairing=N, page=16, pool_token_major=True),
]
