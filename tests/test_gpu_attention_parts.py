"""Work that is dealt in fewer parts than it has units, so that a part has one item's end and the next one's beginning; and batches of more sequences
than a wavefront has lanes: against the oracle in 64 bits."""
import numpy as np
import pytest

from attention_util import orc
from stage_util import f64, torch_mod
from test_gpu_attention import Case
from test_gpu_attention_cache import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    torch = torch_mod()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2311_05827_amd as pkg
    return pkg


def units_and_parts(A, c):
    """Units of places (128; fewer where wide rows leave a workgroup fewer wavefronts), one at least, for every item of `item` rows; and the parts that
    they are dealt in, from the workspace, which has room for two results of an item's rows in each."""
    group, width = c.heads // c.kv, -(-c.head // 32) * 32 if c.head <= 128 else 256
    many = sum(c.new) * group > 32 * len(c.new)
    size = 2 if c.name == "bf16" else 4
    item = 32 if not many else 256 if width // 32 * size <= 8 else 128
    row = (width if width != 96 else 128) * size   # bytes of a tile's row
    unit = 128 if many or row <= 256 else 65536 // row // 2
    units = sum(-(-n * group // item) * max(1, -(-(length + n) // unit)) for length, n in zip(c.contexts, c.new))
    room = A.accept_cache_workspace_size(c.desc)
    return units, room // (c.kv * 2 * item * (width + 2) * 4)


RAGGED = [1500, 3, 2900, 0, 1000]
# contexts, new tokens, heads, key heads, head size, page, words of a tree
CASES = [
    (RAGGED, [1] * 5, 32, 32, 64, 16, 0),
    (RAGGED, [1] * 5, 32, 32, 80, 64, 0),
    (RAGGED, [1, 2, 1, 3, 1], 64, 32, 128, 32, 0),
    (RAGGED[:3], [1] * 3, 16, 16, 256, 64, 0),
    (RAGGED, [40] * 5, 32, 32, 64, 64, 1),
    (RAGGED, [40] * 5, 32, 32, 80, 16, 0),
    ([1200, 2500], [40, 33], 64, 32, 128, 32, 1),
    ([700, 1300, 500], [300, 40, 0], 32, 32, 128, 64, 0),      # more items than one of a sequence
    ([900, 1400], [34, 40], 32, 32, 256, 64, 0),
    ([40 * (s % 9) + s for s in range(70)], [1] * 70, 32, 32, 32, 16, 0),
    ([40 * (s % 9) + s for s in range(70)], [33 + s % 3 for s in range(70)], 32, 32, 32, 16, 0),
    ([400 * (s % 5 == 0) + s for s in range(130)], [2 + 40 * (s % 2) for s in range(130)], 8, 8, 64, 64, 0),
]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("contexts,new,heads,kv_heads,head,page,words", CASES)
def test_parts_with_several_items(A, name, contexts, new, heads, kv_heads, head, page, words):
    c = Cache(A, 1, name, contexts, new, heads, kv_heads, head, page, words=words)
    units, parts = units_and_parts(A, c)
    assert units > 2 * parts
    c.append()
    c.attend()
    c.check_attention()


MANY = {
    "few rows": ([(s * s) % 45 for s in range(600)], [(s % 4) if s % 7 else 0 for s in range(600)]),
    "many rows": ([(s * s) % 45 for s in range(300)], [33 + s % 5 if s % 7 else 0 for s in range(300)]),
    "few of them, few rows": ([(s * s) % 45 for s in range(3000)], [2 * (s % 500 == 7 or s == 2999) for s in range(3000)]),
    "few of them, many rows": ([700 * (s == 1007) for s in range(1025)], [3001 * (s in (0, 1007, 1008, 1024)) for s in range(1025)]),
    "none": ([5] * 100, [0] * 100),
}


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("which", MANY)
def test_more_sequences_than_are_counted(A, name, which):
    """Sequences without new tokens between and behind those with some, tokens behind the last one, and a workspace that holds what was there."""
    torch = torch_mod()
    contexts, new = MANY[which]
    heads = 12 if which.endswith("them, many rows") else 2
    c = Cache(A, 4, name, contexts, new, heads, 1, 16, 16, behind=70)
    many = sum(new) * heads > 32 * len(new)
    assert many == (which.endswith("many rows"))
    c.append()
    c.attend(workspace=torch.full((A.accept_cache_workspace_size(c.desc),), 255, dtype=torch.uint8, device="cuda"))
    assert torch.all(c.o[c.ends[-1]:] == 0)
    c.check_attention()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("new", [9, 70])   # wavefronts with keys of their own, and with keys that they share
def test_a_value_that_some_do_not_see(A, name, new):
    """NaN in one new token's value, in the middle of a part's work."""
    c = Cache(A, 2, name, [1100, 700, 1900], [new] * 3, 32, 32, 80, 16)
    units, parts = units_and_parts(A, c)
    assert units > 2 * parts
    c.append()
    p, at = orc.place(c.table[1], 16, 705)
    c.v_cache[p, :, at, 77] = float("nan")
    o = f64(c.attend())
    assert np.isnan(o[new + 5:2 * new, :, 77]).all()
    o[new + 5:2 * new, :, 77] = 0.0
    assert np.isfinite(o).all()
    c.check_attention()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("q_lengths,k_lengths,which", [([1 + s % 3 for s in range(70)], [1040 + 7 * (s % 30) for s in range(70)], "forward"),
                                                       ([520 + s for s in range(70)], [520 + s for s in range(70)], "backward")])
def test_shares_of_many_sequences(A, name, causal, q_lengths, k_lengths, which):
    c = Case(A, 3, name, q_lengths, k_lengths, 1, 1, 64, causal)
    if which == "forward":
        assert A.accept_attention_workspace_size(c.desc) > 0
    else:
        assert A.accept_attention_backward_workspace_size(c.desc) > 8 * c.nq + 256   # more than the rows' statistics
    c.forward()
    c.check_forward()
    c.check_backward(c.backward())
