"""What the entry points around the block launch, over sizes up to what a card's memory holds: every launch within what a launch can be, and nothing
launched by a call that is refused.  The entry points of a source file run on the host with the launches recorded instead of made."""
from tests.test_launch_sizes_cpu import run

NORM = r"""
static void one()
{
    ss_norm_quant_params q{};
    ss_norm_params& p = q.fwd;
    p.io_dtype = coin(2);
    p.flags = (uint32_t)coin(16) | (coin(2) ? SS_NORM_RMS : 0u);
    p.rows = any(2147418111);
    p.width = any(2 * SS_QUANT_MAX_DIM);
    p.eps = 1e-5f;
    if (2.0 * p.rows * p.width * (p.io_dtype == SS_BF16 ? 2 : 4) > CARD) return;
    p.x = p.residual = p.summed = fake;
    p.weight = p.bias = static_cast<float*>(fake);
    q.q = static_cast<int8_t*>(fake);
    q.scale = static_cast<float*>(fake);
    const int rc = ss_norm_quant(&q, nullptr);
    if ((rc == SS_OK) != (p.width <= SS_QUANT_MAX_DIM)) std::exit(1);
    look(rc, "ss_norm_quant", p.rows, p.width, 0, 0, p.io_dtype, p.flags);
}
"""


def test_norm_quant(tmp_path):
    run(tmp_path, "ss_norm.hip", NORM)


EMBED = r"""
static void one()
{
    ss_embed_bwd_params q{};
    ss_embed_params& p = q.fwd;
    p.table_dtype = coin(2);
    p.io_dtype = coin(2);
    p.flags = (uint32_t)coin(2);
    p.scale = 1.0f;
    p.tokens = any(2147418111);
    p.vocab = 1 + any(2147418110);
    p.dim = 1 + any(65535.0 * 512 - 1);
    const double io = (double)p.tokens * p.dim * (p.io_dtype == SS_BF16 ? 2 : 4), table = (double)p.vocab * p.dim * (p.table_dtype == SS_BF16 ? 2 : 4);
    if (io + table > CARD) return;
    p.ids = p.table = q.dout = fake;
    p.out = q.dtable = q.workspace = fake;
    const int rc = ss_embed_fwd(&p, nullptr);
    if (rc != SS_OK) std::exit(1);
    look(rc, "ss_embed_fwd", p.tokens, p.vocab, p.dim, p.table_dtype, p.io_dtype, p.flags);
    q.workspace_bytes = ss_embed_workspace_bytes(&p);
    const int rb = ss_embed_bwd(&q, nullptr);
    if (rb != SS_OK) std::exit(1);
    look(rb, "ss_embed_bwd", p.tokens, p.vocab, p.dim, p.table_dtype, p.io_dtype, p.flags);
}
"""


def test_embed(tmp_path):
    run(tmp_path, "ss_embed.hip", EMBED)


LOGPROB = r"""
static void one()
{
    ss_logprob_bwd_params q{};
    ss_logprob_params& p = q.fwd;
    p.io_dtype = coin(2);
    p.flags = (uint32_t)coin(2);
    p.rows = any(2147418111);
    p.vocab = 1 + any(2147418110);
    p.top = coin(2) ? coin(65) : 0;
    p.row_stride = p.vocab + coin(100);
    if ((double)p.rows * p.row_stride * (p.io_dtype == SS_BF16 ? 2 : 4) > CARD) return;
    p.logits = p.targets = fake;
    p.logp = p.entropy = p.stats = p.top_logp = static_cast<float*>(fake);
    p.top_ids = static_cast<int64_t*>(fake);
    p.workspace = q.dlogits = fake;
    q.dlogp = q.dentropy = static_cast<float*>(fake);
    p.workspace_bytes = ss_logprob_workspace_bytes(&p);
    const int rc = ss_logprob_fwd(&p, nullptr);
    const int64_t workgroups = p.vocab <= 2048 ? ((int64_t)p.rows + 3) / 4 : (int64_t)p.rows * ((p.vocab + 8191) / 8192);
    if ((rc == SS_OK) != (p.top <= p.vocab && workgroups < (1 << 24))) std::exit(1);
    look(rc, "ss_logprob_fwd", p.rows, p.vocab, p.top, p.row_stride, p.io_dtype, p.flags);
    if (ss_logprob_bwd(&q, nullptr) != rc) std::exit(1);
    look(rc, "ss_logprob_bwd", p.rows, p.vocab, p.top, p.row_stride, p.io_dtype, p.flags);
}
"""


def test_logprob(tmp_path):
    run(tmp_path, "ss_logprob.hip", LOGPROB)


ADAMW = r"""
static void one()
{
    static ss_adamw_tensor list[200];
    ss_adamw_params p{};
    p.state_bits = coin(2) ? 8 : 32;
    p.tensors = coin(200);
    p.beta1 = p.beta2 = 0.9;
    p.count = static_cast<int32_t*>(fake);
    p.list = list;
    double n = 0;
    for (int k = 0; k < p.tensors; ++k) {
        ss_adamw_tensor& t = list[k];
        t = {};
        t.n = (int64_t)any(2147483647) * (coin(20) ? 1 : 1 + coin(60)) * (coin(10) ? 1 : 0);
        if (n + (double)t.n > CARD / (p.state_bits == 8 ? 6 : 12)) t.n = 0;
        n += (double)t.n;
        t.param_dtype = coin(2);
        t.grad_dtype = coin(2);
        t.param = t.m = t.v = fake;
        t.grad = fake;
        t.m_scale = t.v_scale = static_cast<float*>(fake);
    }
    const int rc = ss_adamw_step(&p, nullptr);
    if (rc != SS_OK || launches.empty() || launches.size() > (size_t)p.tensors / 24 + 1) std::exit(1);
    look(rc, "ss_adamw_step", p.tensors, p.state_bits, 0, 0, 0, 0);
}
"""


def test_adamw(tmp_path):
    run(tmp_path, "ss_adamw.hip", ADAMW)
