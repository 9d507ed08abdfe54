"""The native issue of the paged calls (csrc/thk_call.cpp): what it takes, what it leaves to the Python code, and that both ways of
issuing a call are the same call."""
import ctypes

import pytest
import torch

import paper_2407_21018_amd as thk
from paper_2407_21018_amd import binding
from helpers import ws_tensor

L, B, N_q, N_kv, D, S, T, CAP = 1, 2, 8, 2, 128, 200, 64, 32
U = L * B * N_kv


def _calls(device, seed=0):
    """name -> (native function, public function, arguments by name), in an order in which they can be issued."""
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *d: torch.randn(*d, generator=g).to(torch.bfloat16).to(device)  # noqa: E731
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device=device)          # noqa: E731
    shape, pages = thk.make_shape(L, B, N_q, N_kv, D, S, 1, T, 0, thk.THK_BF16, 0), thk.make_pages(4, 64, 4, 9)
    idx = torch.rand(U, D, generator=g).argsort(-1)[:, :T].sort(-1).values.to(torch.int16).contiguous().to(device)
    table = torch.tensor([[3, 0, 7, 5], [8, 1, 2, 4]], dtype=torch.int32, device=device)
    pool = torch.zeros(thk.thk_paged_pool_bytes(shape, pages), dtype=torch.uint8, device=device)
    ws = torch.zeros(thk.thk_workspace_bytes(shape, thk.THK_OP_DECODE_PAGED), dtype=torch.uint8, device=device)
    kt, vt, n = rnd(U, CAP, D), rnd(U, CAP, D), ints(S, 130)
    zeros = lambda *d: torch.zeros(*d, dtype=torch.bfloat16, device=device)      # noqa: E731
    thk.load()
    c = binding._call
    return {
        "paged_write": (c.paged_write, thk.thk_paged_write, dict(
            shape=shape, pages=pages, k=rnd(U, S, D), v=rnd(U, S, D), src_rows=S, n_rows=n, row0=None, idx=idx, table=table, pool=pool, stream=None)),
        "paged_read": (c.paged_read, thk.thk_paged_read, dict(
            shape=shape, pages=pages, pool=pool, table=table, row0=None, n_rows=n, k_out=zeros(U, S, T), v_out=zeros(U, S, D), out_rows=S, stream=None)),
        "tail_append_ragged": (c.tail_append_ragged, thk.thk_tail_append_ragged, dict(
            shape=shape, k_new=rnd(U, 3, D), v_new=rnd(U, 3, D), src_rows=3, src_row0=None, n_new=ints(3, 1), k_tail=kt, v_tail=vt, s_tail=ints(0, 20),
            s_tail_cap=CAP, stream=None)),
        "decode_attn_paged": (c.decode_attn_paged, thk.thk_decode_attn_paged, dict(
            shape=shape, pages=pages, q=rnd(B, N_q, D), pool=pool, table=table, s_pages=n, idx=idx, k_tail=kt, v_tail=vt, s_tail=ints(3, 21),
            s_tail_cap=CAP, out=zeros(B, N_q, D), ws=ws, stream=None)),
    }


def _outputs(calls):
    a = {n: args for n, (_, _, args) in calls.items()}
    return [a["paged_write"]["pool"], a["paged_read"]["k_out"], a["paged_read"]["v_out"], a["tail_append_ragged"]["k_tail"],
            a["tail_append_ragged"]["v_tail"], a["decode_attn_paged"]["out"]]


def test_tensors_on_the_host_are_left_to_the_python_code():
    """... which refuses them."""
    try:
        for name, (native, public, args) in _calls("cpu").items():
            args["stream"] = 0
            for getters in (None, (lambda device: 0, lambda: 0)):
                binding._forget_runtime()
                if getters is not None:
                    binding._call.stream_getters(*getters)
                assert native(*args.values()) == -1
                assert native(*list(args.values())[:-1]) == -1
                with pytest.raises(ValueError, match="must be on the current GPU"):
                    public(*args.values())
    finally:
        binding._forget_runtime()


@pytest.mark.parametrize("other", [bytes, bytearray, lambda s: memoryview(bytes(s)), lambda s: None])
def test_only_pages_are_pages(other):
    for name, (native, public, args) in _calls("cpu").items():
        for which in {"shape", "pages"} & set(args):
            bad = dict(args)
            bad[which] = other(args[which])
            assert native(*bad.values()) == -1
            with pytest.raises((TypeError, ctypes.ArgumentError, AttributeError)):
                public(*bad.values())


class _Sub(torch.Tensor):
    pass


class _Watched:
    def __init__(self, module):
        self.module, self.returned = module, []

    def __getattr__(self, name):
        f = getattr(self.module, name)

        def call(*a):
            st = f(*a)
            self.returned.append((name, st))
            return st
        return call


@pytest.mark.gpu
@pytest.mark.parametrize("side_stream", [False, True])
def test_both_ways_of_issuing_a_call_agree(side_stream, monkeypatch):
    st = torch.cuda.Stream() if side_stream else torch.cuda.current_stream()
    plain, addresses = _calls("cuda"), _calls("cuda")
    names = list(plain)
    thk.thk_paged_read(*_calls("cuda", 1)["paged_read"][2].values())   # the first call of a process sets the stream getters
    watched = _Watched(binding._call)
    monkeypatch.setattr(binding, "_call", watched)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        for name in names:
            plain[name][1](*plain[name][2].values())
        assert watched.returned == [(n, 0) for n in names]            # taken, and issued
        watched.returned.clear()
        for name in names:
            a = {k: v.data_ptr() if isinstance(v, torch.Tensor) and k != "ws" else v for k, v in addresses[name][2].items()}
            addresses[name][1](*a.values())
        assert watched.returned == [(n, -1) for n in names]           # addresses are left to the Python code
    torch.cuda.synchronize()
    for x, y in zip(_outputs(plain), _outputs(addresses)):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert all(x.view(torch.uint8).max() > 0 for x in _outputs(plain))


BAD = [("k", lambda x: x.float()), ("k", lambda x: x[:, ::2]), ("v", lambda x: x[:1]), ("v", lambda x: x.cpu()), ("n_rows", lambda x: x.long()),
       ("n_rows", lambda x: x[:1]), ("idx", lambda x: x.int()), ("table", lambda x: x[:, :3].contiguous()), ("table", lambda x: x.t()),
       ("pool", lambda x: x[:-1]), ("k_out", lambda x: x[:, :-1].contiguous()), ("v_out", lambda x: x.half()),
       ("k_new", lambda x: x[:, :2].contiguous()), ("n_new", lambda x: x.float()), ("k_tail", lambda x: x.transpose(1, 2)),
       ("v_tail", lambda x: x[:, :31].contiguous()), ("s_tail", lambda x: x[:1]), ("s_pages", lambda x: x.to(torch.int16)), ("q", lambda x: x[:, :7]),
       ("out", lambda x: x.float())]


@pytest.mark.gpu
@pytest.mark.parametrize("name,make", BAD, ids=[f"{n}{i}" for i, (n, _) in enumerate(BAD)])
def test_other_tensors_are_refused_by_both(name, make):
    reached = 0
    for call, (native, public, args) in _calls("cuda").items():
        if name not in args:
            continue
        reached += 1
        before = [x.clone() for x in _outputs({**_calls("cuda"), call: (native, public, args)})]
        bad = dict(args)
        bad[name] = make(args[name])
        assert native(*bad.values()) == -1
        with pytest.raises(ValueError):
            public(*bad.values())
        torch.cuda.synchronize()
        for x, y in zip(_outputs({**_calls("cuda"), call: (native, public, args)}), before):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert reached


@pytest.mark.gpu
@pytest.mark.parametrize("name,make", [("q", lambda x: x.as_subclass(_Sub)), ("pool", lambda x: x.view(torch.int32))])
def test_other_forms_are_left_to_the_python_code(name, make):
    """... which takes these: a subclass, a pool of any type that is large enough."""
    native, public, args = _calls("cuda")["decode_attn_paged"]
    want = torch.zeros_like(args["out"])
    public(*{**args, "out": want}.values())
    args[name] = make(args[name])
    assert native(*args.values()) == -1
    public(*args.values())
    torch.cuda.synchronize()
    assert torch.equal(args["out"].view(torch.uint8), want.view(torch.uint8))


@pytest.mark.gpu
def test_workspaces_are_checked_by_both():
    native, public, args = _calls("cuda")["decode_attn_paged"]
    args["shape"].n_split = 3
    n = thk.thk_workspace_bytes(args["shape"], thk.THK_OP_DECODE_PAGED)
    for bad in (torch.empty(n, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(n),
                torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2], (torch.empty(n, dtype=torch.uint8), n),
                (torch.empty(n - 1, dtype=torch.uint8, device="cuda"), n)):
        assert native(*{**args, "ws": bad}.values()) == -1
        with pytest.raises(ValueError, match="ws "):
            public(*{**args, "ws": bad}.values())
    for short in (None, torch.empty(n - 1, dtype=torch.uint8, device="cuda")):
        with pytest.raises(thk.ThkError) as e:
            public(*{**args, "ws": short}.values())
        assert e.value.status == 5
    outs = []
    for ws in (torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(-(-n // 4), device="cuda"), (torch.empty(n, dtype=torch.uint8, device="cuda"), n)):
        outs.append(torch.zeros_like(args["out"]))
        public(*{**args, "ws": ws, "out": outs[-1]}.values())
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.gpu
def test_two_graphs_share_a_workspace():
    """Two captured calls of different sizes with one workspace, replayed in turn on one stream: each has its own answer, every time."""
    torch.manual_seed(3)
    shapes, outs, ones = [], [], []
    big = thk.make_shape(1, 8, 32, 8, D, 9000, 1, T, 0, thk.THK_BF16, 0)     # cut by the lengths on the device
    small = thk.make_shape(1, 1, 32, 8, D, 3000, 1, T, 0, thk.THK_BF16, 0)
    ws = ws_tensor(max(thk.thk_workspace_bytes(s, thk.THK_OP_DECODE_PAGED) for s in (big, small)))
    for s in (big, small):
        n_pages = -(-s.S // 128)
        pages = thk.make_pages(8, 128, n_pages, n_pages * s.B)
        pool = torch.zeros(thk.thk_paged_pool_bytes(s, pages), dtype=torch.uint8, device="cuda")
        units = s.B * s.N_kv
        idx = torch.rand(units, D, device="cuda").argsort(-1)[:, :T].sort(-1).values.to(torch.int16).contiguous()
        table = torch.randperm(n_pages * s.B, device="cuda").to(torch.int32).view(s.B, n_pages).contiguous()
        rows = torch.tensor([s.S - 700 * b for b in range(s.B)], dtype=torch.int32, device="cuda")
        k, v = (torch.randn(units, s.S, D, device="cuda").to(torch.bfloat16) for _ in range(2))
        thk.thk_paged_write(s, pages, k, v, s.S, rows, None, idx, table, pool)
        q = torch.randn(s.B, s.N_q, D, device="cuda").to(torch.bfloat16)
        out = torch.zeros_like(q)
        ones.append((s, pages, q, pool, table, rows, idx, None, None, None, 0, out, ws))
        outs.append(out)
    wants, graphs = [], []
    for args in ones:
        thk.thk_decode_attn_paged(*args)
        torch.cuda.synchronize()
        wants.append(args[11].clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            thk.thk_decode_attn_paged(*args)
        graphs.append(graph)
    for i in range(6):
        for out in outs:
            out.zero_()
        ws.fill_(255)
        for which in ((0, 1), (1, 0), (0, 1, 0))[i % 3]:
            graphs[which].replay()
        if i % 2:
            torch.cuda.synchronize()
        for out, want in zip(outs, wants):
            assert torch.equal(out, want)
