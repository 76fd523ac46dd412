"""One turn of the loop around the verifier: registers are drawn under masks of occupied ones, the candidates checked, the draws scored, the verdicts
made a loss, its gradient taken to the logits and on to a small head's weights, and those gradients clipped."""
import numpy as np
import pytest

from paper_2506_17506_b200 import synth

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2506_17506_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_turn_of_the_loop(B, dtype):
    import torch
    import oracle
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    wl = synth.workload(1)
    prog = synth.build_program(wl.shapes[0], wl.seeds[0])
    seed_rows, _ = synth.candidate_rows(prog, 4, 0.0, wl.seeds[0])
    S, P = 24, prog.P
    instr = np.repeat(np.arange(prog.n_instrs), prog.instr_n_defs)
    col = np.concatenate([np.arange(o, o + d) for o, d in zip(prog.instr_op_off[:-1], prog.instr_n_defs)]).astype(np.int64)
    vreg = prog.op_vreg[col]
    D = len(col)
    gp = B.Program(prog)
    gp.vl_liveness()
    masks = gp.vl_occupied_masks(torch.from_numpy(seed_rows[0].view(np.int16)).cuda().view(torch.uint16), P, words=True)
    gen = torch.Generator(device="cuda").manual_seed(7)
    hidden = torch.randn(S * D, 48, generator=gen, device="cuda").to(kind)
    head = torch.randn(P, 48, generator=gen, device="cuda").to(kind)
    logits = hidden @ head.t()
    which = torch.from_numpy(instr.astype(np.int32)).cuda().repeat(S)
    widths = torch.from_numpy(prog.vreg_width[vreg]).cuda().repeat(S)
    args = dict(occupied=masks, mask_rows=which, widths=widths, scale=0.2)
    u = torch.rand(S * D, generator=gen, device="cuda")
    drawn = B.vl_token_sample(logits, u, top_p=0.95, token_dtype=torch.uint16, **args)
    # every register that was drawn is free for the whole tuple, and is scored as the draw says
    tok = drawn.tokens.to(torch.int32).cpu().numpy().reshape(S, D)
    shut = gp.vl_occupied_masks(torch.from_numpy(seed_rows[0].view(np.int16)).cuda().view(torch.uint16), P)
    for j in range(D):
        w = int(prog.vreg_width[vreg[j]])
        free = [r for r in range(P - w + 1) if not shut[instr[j], r:r + w].any()]
        assert set(tok[:, j].tolist()) <= (set(free) if free else {65535})
    sc = B.vl_token_logprobs(logits, drawn.tokens, **args)
    there = torch.from_numpy((tok.reshape(-1) != 65535)).cuda()
    assert bool(((sc.logprob - drawn.logprob).abs()[there] <= 64 * U * (1 + drawn.logprob.abs()[there])).all())
    assert bool((drawn.drawn_logprob >= drawn.logprob).all())
    # candidates: every occurrence of a register's value carries what its first definition drew
    rows = np.zeros((S, gp.pitch), dtype=np.uint16)
    first = {int(v): j for j, v in reversed(list(enumerate(vreg)))}
    place = np.array([first[int(v)] for v in prog.op_vreg])
    rows[:, :prog.n_operands] = np.where(tok == 65535, 0, tok)[:, place]
    out = gp.vl_verify(torch.from_numpy(rows.view(np.int16)).cuda().view(torch.uint16))
    op = oracle.OracleProgram(prog)
    assert B.verdicts_to_numpy(out).tobytes() == op.verify(op.liveness(), rows).tobytes()
    loss, _, g = B.vl_policy_loss([out], torch.arange(0, S * D + 1, D, device="cuda"), sc.logprob, drawn.logprob, pair_cost=0.01)
    assert bool(torch.isfinite(loss))
    dlogits = B.vl_token_logprobs_backward(logits, drawn.tokens, sc.row_stats, g, **args)
    grads = [(dlogits.t().float() @ hidden.float()).to(kind), dlogits.float().sum(0)]
    before = [x.double() for x in grads]
    norm = float(torch.sqrt(sum((x * x).sum() for x in before)))
    got = B.vl_clip_grads(grads, norm / 2)
    assert abs(float(got.norm) - norm) <= 8 * U * norm and abs(float(got.factor) - 0.5) <= 8 * U
    half = {"f32": U, "bf16": 2.0 ** -8}
    for b, x in zip(before, grads):
        assert bool(((x.double() - b / 2).abs() <= (8 * U + half["f32" if x.dtype == torch.float32 else "bf16"]) * b.abs() + 2.0 ** -133).all())
    gp.close()
