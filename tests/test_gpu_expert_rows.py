"""The rows of a routed layer by expert against a stable sort: whole numbers, equal."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_35481_amd import ffn  # noqa: E402

DEV = torch.device("cuda:0")


def want(ids, L, slot):
    of = ids.reshape(-1).long()
    E = L if slot is None else len(slot)
    there = torch.arange(L) if slot is None else slot.long()
    of = torch.where((of >= 0) & (of < E), there[of.clamp(0, E - 1)], -1)
    of = torch.where((of >= 0) & (of < L), of, L)
    order = torch.sort(of, stable=True).indices
    count = torch.bincount(of, minlength=L + 1)[:L]
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), count.cumsum(0)])
    pairs = torch.where(torch.arange(len(of)) < offsets[-1], order, -1)
    places = torch.full((len(of),), -1)
    places[order[:offsets[-1]]] = torch.arange(int(offsets[-1]))
    return offsets.int(), pairs.int(), places.view(ids.shape).int()


def check(ids, L, slot):
    got = ffn.expert_rows(ids.to(DEV), L, expert_slot=None if slot is None else slot.to(DEV))
    for g, w, name in zip(got, want(ids, L, slot), ("offsets", "pairs", "places")):
        assert g.dtype == torch.int32 and torch.equal(g.cpu(), w), name


@pytest.mark.parametrize("T,k,E,L", [(1, 1, 1, 1), (1, 8, 128, 128), (63, 1, 3, 2), (64, 2, 16, 16), (1023, 8, 37, 37),
                                     (1024, 8, 1024, 1024), (1025, 8, 1000, 512), (4097, 2, 64, 1), (8192, 1, 2, 2),
                                     (8193, 1, 5, 5), (20000, 4, 256, 200), (70001, 8, 640, 513), (300000, 2, 8, 8)])
def test_rows(T, k, E, L):
    g = torch.Generator().manual_seed(T)
    ids = (torch.rand((T, k), generator=g) ** 2 * E).long().clamp(max=E - 1).int()
    slot = torch.full((E,), -1, dtype=torch.int32)
    slot[torch.randperm(E, generator=g)[:L]] = torch.arange(L, dtype=torch.int32)
    check(ids, L, slot)
    check(ids, L, None)                   # ids from L on are nowhere


@pytest.mark.parametrize("T", [50, 9000])
def test_ids_and_slots_that_are_nowhere(T):
    g = torch.Generator().manual_seed(T)
    ids = torch.randint(-3, 12, (T, 3), generator=g).int()
    ids[0] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0])
    check(ids, 6, torch.tensor([0, 5, 5, -1, 6, 2 ** 31 - 1, -2 ** 31, 1], dtype=torch.int32))
    check(torch.full((T, 3), 7, dtype=torch.int32), 8, None)
    check(torch.full((T, 3), -1, dtype=torch.int32), 8, None)


def test_no_tokens():
    got = ffn.expert_rows(torch.zeros((0, 4), dtype=torch.int32, device=DEV), 5)
    assert torch.equal(got[0].cpu(), torch.zeros(6, dtype=torch.int32)) and got[1].numel() == 0


def test_refusals():
    ids = torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(TypeError):
        ffn.expert_rows(ids.long(), 4)
    with pytest.raises(ValueError):
        ffn.expert_rows(ids.t(), 4)
    with pytest.raises(TypeError):
        ffn.expert_rows(ids, 4, expert_slot=torch.zeros(8, dtype=torch.int64, device=DEV))
    with pytest.raises(TypeError):
        ffn.expert_rows(ids, 4, expert_slot=torch.zeros(8, dtype=torch.int32))
    for L in (0, -1, 1025):
        with pytest.raises(Exception, match="topoep_expert_rows"):
            ffn.expert_rows(ids, L)
    with pytest.raises(TypeError):
        ffn.expert_rows(ids, 4.0)
