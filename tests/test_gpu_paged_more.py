"""The cases of paged_more on the GPU, checked as test_gpu_paged checks its own."""
import pytest
import torch

import paged_more as more
import paged_util as u
import test_gpu_paged as t
from paper_2602_08686_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("c", more.ROWS, ids=range(len(more.ROWS)))
def test_rows_are_transformed_and_find_their_pages(c):
    t.test_rows_are_transformed_and_find_their_pages(c)


@pytest.mark.parametrize("c", more.MANY, ids=range(len(more.MANY)))
def test_attention_over_pages(c):
    t.test_attention_over_pages(c)


@pytest.mark.parametrize("kind", ["bad_pages", "beyond", "masked_infinity", "masked_nan", "one_component"])
@pytest.mark.parametrize("c", [more.MANY[0], more.MANY[1], more.MANY[5], more.MANY[7]], ids=range(4))
def test_what_is_not_seen_has_no_influence(c, kind):
    t.test_what_is_not_seen_has_no_influence(c, kind)


def test_a_tensor_on_the_host_is_refused():
    """... by its name, wherever the others are, before anything is launched."""
    c = u.case(n=3, lengths=((20, 20), (9, 9)), counts=((3, 3), (3, 1)), norm=True, rot_dim=64)
    good = t.on_gpu(c, u.make(c))
    rot, q_out, k_out, out = u.rotation(c), t.nines(c, 8), t.nines(c, 2), t.nines(c, 8)
    lse = torch.full((2, 8, 3), 9.0, device="cuda")
    for name in ("q", "k", "v", "k_pages", "v_pages", "table", "length", "count", "positions", "inv_freq", "q_weight", "k_weight"):
        x = dict(good, **{name: good[name].cpu() if name[1:] != "_pages" else torch.empty_like(good[name], device="cpu")})
        calls = {
            "rotate": lambda: B.ckv_norm_rotate(x["params"], rot, x["q"], x["k"], x["positions"], x["inv_freq"], x["q_weight"], x["k_weight"], q_out, k_out,
                                                count=x["count"]),
            "append": lambda: B.ckv_paged_append(x["params"], rot, x["pages"], x["k"], x["v"], x["k_pages"], x["v_pages"], x["table"], x["length"],
                                                 count=x["count"], positions=x["positions"], inv_freq=x["inv_freq"], k_weight=x["k_weight"], q=x["q"],
                                                 q_weight=x["q_weight"], q_out=q_out),
            "attend": lambda: B.ckv_paged_attention(x["params"], x["pages"], x["q"], x["k_pages"], x["v_pages"], x["table"], x["length"], x["n_rows"], out,
                                                    lse, x["ws"], count=x["count"])}
        takes = {"rotate": ("q", "k", "count", "positions", "inv_freq", "q_weight", "k_weight"), "append": tuple(good),
                 "attend": ("q", "k_pages", "v_pages", "table", "length", "count")}
        for call in calls:
            if name in takes[call]:
                with pytest.raises(ValueError, match=f"^{name} has to be on the GPU"):
                    calls[call]()
    torch.cuda.synchronize()
    for x in (q_out, k_out, out, lse):
        assert (x == 9.0).all()
