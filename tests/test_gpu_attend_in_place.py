"""fastav_attend in a loop that changes lengths, page tables, query bounds and queries in place between calls that follow one another without a pause."""
import pytest
import torch

from paper_2601_13143_b200 import fastav
from test_gpu_attend import Problem, _cu

pytestmark = pytest.mark.gpu

SHAPES = {
    # few rows only, many rows only, both side by side (with more and with fewer prefixes)
    "few": dict(hq=28, hkv=4, dim=128, lens=[700, 90, 1500, 333], rows=[1, 2, 1, 2]),
    "many": dict(hq=16, hkv=4, dim=128, lens=[700, 300, 250], rows=[12, 40, 33]),
    "both": dict(hq=32, hkv=8, dim=128, lens=[60, 130, 77, 200, 45, 66], rows=[1] * 6, prefix_lens=[1500], groups=[0, 6]),
    "both_two_prefixes": dict(hq=28, hkv=4, dim=64, lens=[60, 130, 77, 200, 45, 66], rows=[2, 1, 2, 1, 2, 2], prefix_lens=[1100, 700], groups=[0, 3, 6]),
}


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("name", SHAPES)
def test_what_changes_in_place_between_calls_is_seen(name, graph):
    p = Problem(fmt="int8", page=32, seed=40, **SHAPES[name])
    turns, batch, n_prefix = 12, len(p.lens), len(p.prefix_lens)
    gen = torch.Generator().manual_seed(41)
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731

    def shuffled(table, lens):  # the full pages of a row in another order (the last one, which is not full, stays)
        table = table.clone()
        for b, n in enumerate(lens):
            full = n // p.page
            table[b, :full] = table[b, torch.randperm(full, generator=gen)]
        return table

    states = []
    for _ in range(turns):
        lens = [max(r, n - int(torch.randint(0, 3, (1,), generator=gen)) * p.page) for n, r in zip(p.lens, p.rows)]
        rows = [p.rows[i] for i in torch.randperm(batch, generator=gen)]
        states.append(dict(lens=dev(lens), table=shuffled(p.tables[0], p.lens).cuda(), cu=_cu(rows).cuda(),
                           q=torch.randn(p.total, p.hq, p.dim, generator=gen).to(torch.bfloat16).cuda(),
                           plens=dev([n - 32 * int(torch.randint(0, 20, (1,), generator=gen)) for n in p.prefix_lens] or [0]),
                           ptable=shuffled(p.tables[1], p.prefix_lens).cuda()))
    live = {k: torch.empty_like(v) for k, v in states[0].items()}
    params = p.params(max_qlen=max(p.rows), max_prefix_q=p.total if n_prefix else 0)
    ws = torch.full((fastav.fastav_attend_workspace_bytes(params, p.cache),), 0xFF, dtype=torch.uint8, device="cuda")
    outs = [(torch.full_like(p.out, 9.0), torch.full_like(p.lse, 9.0)) for _ in range(turns)]
    groups = dev(p.groups)

    def call(i, state):
        for k, v in live.items():
            v.copy_(state[k], non_blocking=True)
        more = dict(cu_prefix=groups, prefix_table=live["ptable"], prefix_lens=live["plens"]) if n_prefix else {}
        fastav.fastav_attend(params, p.cache, live["q"], live["cu"], live["table"], live["lens"], outs[i][0], ws, lse_out_opt=outs[i][1], device_status=p.status, **more)

    alone = []
    for i, state in enumerate(states):
        call(i, state)
        torch.cuda.synchronize()
        alone.append((outs[i][0].clone(), outs[i][1].clone()))
        outs[i][0].fill_(9.0)
        outs[i][1].fill_(9.0)
    torch.cuda.synchronize()
    assert len({float(lse.sum()) for _, lse in alone}) == turns   # every turn asks for something else
    if graph:
        side, recorded = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(recorded, stream=side):
            for i, state in enumerate(states):
                call(i, state)
        for _ in range(3):
            recorded.replay()
    else:
        for _ in range(3):
            for i, state in enumerate(states):
                call(i, state)
    torch.cuda.synchronize()
    for (out, lse), (want, wlse) in zip(outs, alone):
        assert torch.equal(out, want) and torch.equal(lse, wlse)
    assert int(p.status) == 0
