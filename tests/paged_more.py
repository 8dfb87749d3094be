"""Further cases of the paged cache's calls: those that reach the kernels' instances and plans that the shorter ones do not."""
import paged_util as u

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
