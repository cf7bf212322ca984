// Selective state space scan: entry points, and the rules by which a call is cut into blocks and segments.
#include <cuda_runtime.h>

#include <cstdint>

#include "mebptt.h"
#include "scan.hpp"
#include "scan_kernels.hpp"

using namespace mebptt::seq;

namespace {

// Steps of a segment and their number, for a kernel of `blocks` blocks a segment where `room` are wanted: as many as the device holds
// at once, backward twice that.  Segments cost a kernel in front that walks the steps once more (backward: a lighter one, and more
// sums to join), so that fewer than `least` of them lose by it; a segment begins where a state is kept and has 16 steps at least;
// there are 64 at most (each block folds what the others hand it).
// Measured in us, 512 steps of 1024 channels of 16 states in bf16, all kernels of the pass, with 1, 2, 3, 4 and 6 segments.
// Forward: 32 rows (wanted 2) 157, 177, 187, 185, 195; 20 rows (wanted 3) 130, 137, 134, 126, 127; 16 rows (wanted 4) 109, 113, 116,
// 103, 107; 10 rows (wanted 6) 108, 99, 87, 78, 79.
// Backward: 32 rows (wanted 2) 420, 434, 451, 445, 440; 20 rows (wanted 3) 338, 342, 296, 300, 286; 16 rows (wanted 4) 269, 251, 246,
// 238, 240; 10 rows (wanted 7) 265, 208, 178, 184, 166.
// Backward with as many blocks as the device holds against twice that: 13 rows of 161 steps of 300 channels of 10 states in bf16
// 49 and 43, but 4 rows of 2000 steps of 512 channels of 16 states in fp32 173 and 180.
void cut(int64_t t, int64_t blocks, int64_t room, int least, int spacing, int& segment, int& segments) {
  const int64_t unit = spacing > 16 ? spacing : 16;
  int64_t n = room / blocks;
  if (n > (t + unit - 1) / unit) n = (t + unit - 1) / unit;
  if (n > 64) n = 64;
  if (n < least) n = 1;
  int64_t len = (t + n - 1) / n;
  len = (len + unit - 1) / unit * unit;
  segment = (int)len;
  segments = (int)((t + len - 1) / len);
}

constexpr int SMS = 148;        // what the rules count on: workspaces must not depend on the device a call finds

struct Cut {
  int np, blocks_f, blocks_b;
  int segment_f, segments_f, segment_b, segments_b;
};

bool check(const mebptt_scan_desc* d, ScanArgs& a, Cut& c) {
  if (!d || d->batch < 1 || d->channels < 1 || d->states < 1 || d->states > 64 || d->groups < 1 || d->t < 1 || d->t > (1 << 30)) return false;
  if (d->channels > (1 << 24) || d->batch > (1 << 24) || d->channels % d->groups || d->reserved || !valid_dtype(d->dtype)) return false;
  if ((d->flags & ~MEBPTT_SCAN_SOFTPLUS) || (d->spacing != 8 && d->spacing != 16 && d->spacing != 32)) return false;
  const int64_t gn = (int64_t)d->groups * d->states;
  if (!places(d->u_step, d->u_row, d->t, d->batch, d->channels, a.pu) || !places(d->delta_step, d->delta_row, d->t, d->batch, d->channels, a.pd) ||
      !places(d->z_step, d->z_row, d->t, d->batch, d->channels, a.pz) || !places(d->y_step, d->y_row, d->t, d->batch, d->channels, a.py) ||
      !places(d->b_step, d->b_row, d->t, d->batch, gn, a.pb) || !places(d->c_step, d->c_row, d->t, d->batch, gn, a.pc))
    return false;
  a.batch = d->batch; a.channels = d->channels; a.states = d->states; a.groups = d->groups; a.gchannels = d->channels / d->groups;
  a.t = (int)d->t; a.spacing = d->spacing; a.softplus = d->flags & MEBPTT_SCAN_SOFTPLUS;
  const int lanes = scan_lanes(d->states), chf = scan_fwd_channels(lanes), chb = scan_bwd_channels(lanes);
  c.np = 8 * lanes;
  c.blocks_f = (a.gchannels + chf - 1) / chf;
  c.blocks_b = (a.gchannels + chb - 1) / chb;
  const bool half = d->dtype == MEBPTT_BF16;
  cut(d->t, (int64_t)d->groups * c.blocks_f * d->batch, SMS * scan_fwd_blocks(lanes, half), 4, d->spacing, c.segment_f, c.segments_f);
  cut(d->t, (int64_t)d->groups * c.blocks_b * d->batch, 2 * SMS * scan_bwd_blocks(lanes, half, d->spacing), 3, d->spacing, c.segment_b, c.segments_b);
  return true;
}
// What a grid can count, and backward a row of sums over channels (both halves of every group's states) in 32 bits.
bool fits(const mebptt_scan_desc* d, const Cut& c, bool back) {
  return d->batch <= 65535 && (!back || (int64_t)d->groups * 2 * c.np <= INT32_MAX) &&
         (double)d->t * d->batch * d->groups * 2 * c.np / 256 + (double)d->channels * (d->states + 2) / 32 < 2e9;
}

size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// The workspace: what segments begin with, and for the backward pass the sums of blocks and rows.
struct Work {
  size_t ends, dts, bc, pa, pd, pb, bytes;
};
Work work(const mebptt_scan_desc* d, const Cut& c, bool back) {
  Work w = {};
  const size_t bd = (size_t)d->batch * d->channels;
  const int segments = back && c.segments_b > c.segments_f ? c.segments_b : c.segments_f;
  size_t at = 0;
  if (segments > 1) {
    w.ends = at; at += up((size_t)(segments + 1) * bd * c.np * 4);
    w.dts = at; at += up((size_t)segments * bd * 4);
  }
  if (back) {
    w.bc = at; at += up((size_t)c.blocks_b * d->t * d->batch * d->groups * 2 * c.np * 4);
    w.pa = at; at += up((size_t)c.segments_b * bd * c.np * 4);
    w.pd = at; at += up((size_t)c.segments_b * bd * 4);
    w.pb = at; at += up((size_t)c.segments_b * bd * 4);
  }
  w.bytes = at;
  return w;
}

// Whether groups of eight channels, and of four states, load as one.
void vectors(const mebptt_scan_desc* d, ScanArgs& a) {
  const size_t e = elem_size(d->dtype);
  const void* const u[] = {a.u, a.du};
  const void* const dl[] = {a.delta, a.ddelta};
  const void* const zs[] = {a.z, a.dz};
  const void* const ys[] = {a.y, a.dy};
  bool v = a.groups == 1 || a.gchannels % 8 == 0;
  for (const void* p : u) v = v && aligned(p, a.pu, 8, e);
  for (const void* p : dl) v = v && aligned(p, a.pd, 8, e);
  if (a.z)
    for (const void* p : zs) v = v && aligned(p, a.pz, 8, e);
  for (const void* p : ys) v = v && aligned(p, a.py, 8, e);
  a.vec_d = v;
  const Places none{0, 0};
  const void* const fs[] = {a.A, a.s_in, a.s_out, a.ds_out, a.ds_in};
  bool s = a.states % 4 == 0 && aligned(a.B, a.pb, 4, e) && aligned(a.C, a.pc, 4, e);
  for (const void* p : fs) s = s && aligned(p, none, 4, 4);
  a.vec_s = s;
}

bool naturals(const ScanArgs& a, int dtype) {
  const size_t e = elem_size(dtype);
  const void* const typed[] = {a.u, a.delta, a.z, a.B, a.C, a.dy, a.y, a.du, a.ddelta, a.dz};
  const void* const floats[] = {a.A, a.skip, a.bias, a.s_in, a.ds_out, a.s_out, a.ds_in, a.lengths};
  for (const void* p : typed)
    if (!natural(p, e)) return false;
  for (const void* p : floats)
    if (!natural(p, 4)) return false;
  return !(reinterpret_cast<uintptr_t>(a.kept) & 15);
}

bool workspace_fits(const void* ws, size_t have, size_t need) {
  return need == 0 || (ws && !(reinterpret_cast<uintptr_t>(ws) & 255) && have >= need);
}

}  // namespace

extern "C" {

size_t mebptt_scan_kept_bytes(const mebptt_scan_desc* desc) {
  ScanArgs a = {};
  Cut c;
  if (!check(desc, a, c)) return 0;
  return (size_t)((desc->t + desc->spacing - 1) / desc->spacing) * desc->batch * desc->channels * c.np * 4;
}

size_t mebptt_scan_workspace_bytes(const mebptt_scan_desc* desc, int backward) {
  ScanArgs a = {};
  Cut c;
  if (!check(desc, a, c)) return 0;
  return work(desc, c, backward != 0).bytes;
}

int mebptt_scan_forward(const mebptt_scan_desc* desc, const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                        const float* skip, const void* z, const float* delta_bias, const float* s_in, const int32_t* lengths,
                        void* workspace, size_t workspace_bytes, void* stream, void* y, float* s_out, void* kept) {
  ScanArgs a = {};
  Cut c;
  if (!check(desc, a, c) || !u || !delta || !A || !Bm || !Cm || !y) return MEBPTT_ERR_ARG;
  a.u = u; a.delta = delta; a.A = A; a.B = Bm; a.C = Cm; a.skip = skip; a.z = z; a.bias = delta_bias; a.s_in = s_in; a.lengths = lengths;
  a.y = y; a.s_out = s_out; a.kept = (float*)kept;
  if (!naturals(a, desc->dtype)) return MEBPTT_ERR_ARG;
  if (!fits(desc, c, false)) return MEBPTT_ERR_UNSUPPORTED;
  const Work w = work(desc, c, false);
  if (!workspace_fits(workspace, workspace_bytes, w.bytes)) return MEBPTT_ERR_WORKSPACE;
  a.ends = (float*)((char*)workspace + w.ends);
  a.dts = (float*)((char*)workspace + w.dts);
  a.segment = c.segment_f; a.segments = c.segments_f; a.blocks = c.blocks_f;
  vectors(desc, a);
  if (!scan_forward(a, desc->dtype == MEBPTT_BF16, (cudaStream_t)stream)) return MEBPTT_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? MEBPTT_OK : MEBPTT_ERR_CUDA;
}

int mebptt_scan_backward(const mebptt_scan_desc* desc, const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                         const float* skip, const void* z, const float* delta_bias, const int32_t* lengths, const void* kept,
                         const void* dy, const float* ds_out, void* workspace, size_t workspace_bytes, void* stream, void* du,
                         void* ddelta, float* dA, void* dB, void* dC, float* dskip, void* dz, float* ddelta_bias, float* ds_in) {
  ScanArgs a = {};
  Cut c;
  if (!check(desc, a, c) || !u || !delta || !A || !Bm || !Cm || !kept || !dy || !du || !ddelta || !dA || !dB || !dC || !z != !dz) return MEBPTT_ERR_ARG;
  a.u = u; a.delta = delta; a.A = A; a.B = Bm; a.C = Cm; a.skip = skip; a.z = z; a.bias = delta_bias; a.lengths = lengths;
  a.kept = (float*)kept; a.dy = dy; a.ds_out = ds_out; a.du = du; a.ddelta = ddelta; a.dz = dz; a.ds_in = ds_in;
  const size_t e = elem_size(desc->dtype);
  if (!naturals(a, desc->dtype) || !natural(dB, e) || !natural(dC, e) || !natural(dA, 4) || !natural(dskip, 4) || !natural(ddelta_bias, 4)) return MEBPTT_ERR_ARG;
  if (!fits(desc, c, true)) return MEBPTT_ERR_UNSUPPORTED;
  const Work w = work(desc, c, true);
  if (!workspace_fits(workspace, workspace_bytes, w.bytes)) return MEBPTT_ERR_WORKSPACE;
  char* const ws = (char*)workspace;
  a.ends = (float*)(ws + w.ends); a.dts = (float*)(ws + w.dts);
  a.part_bc = (float*)(ws + w.bc); a.part_a = (float*)(ws + w.pa); a.part_d = (float*)(ws + w.pd); a.part_b = (float*)(ws + w.pb);
  a.segment = c.segment_b; a.segments = c.segments_b;
  vectors(desc, a);
  if (c.segments_b > 1) {
    a.blocks = c.blocks_f;
    if (!scan_adjoints(a, desc->dtype == MEBPTT_BF16, (cudaStream_t)stream)) return MEBPTT_ERR_CUDA;
  }
  a.blocks = c.blocks_b;
  if (!scan_backward(a, desc->dtype == MEBPTT_BF16, dA, dB, dC, dskip, ddelta_bias, (cudaStream_t)stream)) return MEBPTT_ERR_CUDA;
  return cudaGetLastError() == cudaSuccess ? MEBPTT_OK : MEBPTT_ERR_CUDA;
}

}  // extern "C"
