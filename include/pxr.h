/*
 * pxr — batched pixel-observation renderer for one AMD MI355X (gfx950).
 *
 * C ABI of the hot path that PixelBrax (arXiv 2502.00021) moves onto the
 * accelerator: for each of B parallel environments and each of S steps, turn
 * the simulator's rigid-body poses into one small RGB observation without the
 * frame ever leaving the device (paper section 1), optionally with a colour or
 * a video distractor fused into the renderer (paper section 2) and with all
 * randomness drawn from an explicit seeded generator (paper sections 1-2).
 *
 * All functions return a PXR_* status code, never throw or abort across the
 * ABI, and leave out-parameters untouched on error.  pxr_last_error() gives a
 * human-readable reason for the last failure on the calling thread.
 *
 * Pointers named d_* are DEVICE pointers owned by the caller; everything else
 * is host memory.  The library owns only the pxr_scene and the device-side
 * constants it uploads at creation.
 */
#ifndef PXR_H
#define PXR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct pxr_scene pxr_scene; /* opaque, owned by the library */

enum { PXR_OK = 0, PXR_ERR_INVALID_ARG = 1, PXR_ERR_UNSUPPORTED = 2, PXR_ERR_OOM = 3, PXR_ERR_DEVICE = 4 };
enum { PXR_CAPSULE = 0, PXR_SPHERE = 1, PXR_BOX = 2, PXR_MESH = 3 };
enum { PXR_DISTRACT_NONE = 0, PXR_DISTRACT_COLOR = 1, PXR_DISTRACT_VIDEO = 2 };

/* Winning-id values that are not triangles. */
#define PXR_ID_GROUND 0xFFFFFFFEu
#define PXR_ID_BG     0xFFFFFFFFu

/* One rigid body = one primitive, tessellated once at scene creation.
 *   shape: capsule (r,r,r,h): radius r, half-length h of the segment along local +Z
 *          sphere  (r,r,r,0)
 *          box     (ex,ey,ez,0): half-extents
 *          The posed local vertex is (shape[0]*ux, shape[1]*uy, shape[2]*uz + s*shape[3]) for the
 *          unit-shape template vertex (ux,uy,uz) with cap selector s.
 *   n_lon, n_lat: capsule/sphere: longitudes, latitude steps PER HEMISPHERE
 *          (capsule 4*n_lon*n_lat triangles, sphere 2*n_lon*(2*n_lat-1));
 *          box: n_lon = cells per face edge (12*n_lon^2 triangles, checker
 *          colour multiplier 1 / 0.5 per cell), n_lat ignored.
 *   PXR_MESH (the paper names mesh rendering as its renderer's next step): the caller's own triangle mesh.
 *          mesh_verts [n_mesh_verts*3] body-frame positions, used as the template as they are (selector 0,
 *          scaled per axis by shape[0..2], shape[3] ignored); mesh_tris [n_mesh_tris*3] indices into them,
 *          counter-clockwise seen from outside (back faces are culled); mesh_tri_mul [n_mesh_tris] colour
 *          multiplier per triangle, or NULL = 1.  Host arrays, copied at scene creation; ignored for the
 *          other types.  A triangle's normal is the unit cross product of its unscaled vertices (zero for
 *          a triangle without area: it is shaded with the ambient term only). */
typedef struct {
    uint32_t type;
    float shape[4];
    float rgb[3];
    uint32_t n_lon, n_lat;
    const float* mesh_verts;
    const uint32_t* mesh_tris;
    const float* mesh_tri_mul;
    uint32_t n_mesh_verts, n_mesh_tris;
} pxr_body_desc;

/* Scene = what is common to all environments: image size, bodies, camera rig,
 * light, ground, background.  The camera sits at (root body position +
 * cam_offset) in WORLD axes and looks at the root body; pinhole, fov_y_deg
 * vertical field of view.  light_dir points TOWARD the light.  The ground is
 * the plane z = 0 with a two-grey checkerboard of ground_cell metres. */
typedef struct {
    uint32_t width, height, n_bodies, root_body;
    const pxr_body_desc* bodies; /* host, borrowed for the call only */
    float fov_y_deg, cam_offset[3], cam_up[3], z_near, z_far;
    float light_dir[3], ambient, diffuse;
    uint32_t ground_enabled;
    float ground_cell, ground_grey[2];
    float background_rgb[3];
} pxr_scene_desc;

/* Distractor state (paper section 2: the colour kind or the video kind, mutually exclusive).
 *   COLOR: per (env, step) and per channel, scale ~ U[scale_lo,scale_hi) and
 *          offset ~ U[offset_lo,offset_hi) from the counter-based generator
 *          keyed by (seed, env, step); every pixel becomes clamp(c*scale+offset, 0, 1).
 *   VIDEO: d_video is a device-resident uint8 [n_frames,H,W,3] clip; env e at
 *          step t shows frame (env_offset[e] + t) mod n_frames, alpha-blended
 *          onto pixels whose winner is the ground or the background.
 *          d_env_offset: device uint32 [B] (indexed by the env's position in
 *          the batch), or NULL = drawn from the generator.  With n_videos > 1
 *          every environment plays one clip of a set (paper section 2: each
 *          environment gets a clip picked at random), chosen by d_env_video or
 *          drawn from the generator.  All buffers are caller-owned and must stay alive while bound. */
typedef struct {
    uint32_t mode;
    uint64_t seed;
    float scale_lo, scale_hi, offset_lo, offset_hi;
    const uint8_t* d_video;
    uint32_t n_frames;
    float alpha;
    const uint32_t* d_env_offset;
    uint32_t n_videos;            /* VIDEO: 0 or 1 = one clip; > 1: d_video is [n_videos,n_frames,H,W,3] */
    const uint32_t* d_env_video;  /* VIDEO, n_videos > 1: device uint32 [B], the clip of each environment
                                     (values >= n_videos are reduced modulo n_videos), or NULL = drawn */
} pxr_distractor_desc;

/* Build a scene on the current HIP device: validate, tessellate, derive the
 * camera constants, upload (one allocation, one synchronous copy).  Host only,
 * not on the hot path.  (Paper section 1: an environment is a set of rigid bodies seen by a camera; the
 * paper gives no geometry, camera or lighting model, so primitives, tessellation, the root-tracking pinhole
 * camera and the flat Lambert-plus-ambient light are this library's reading of "rendered from the
 * simulator's state".)
 * Errors: INVALID_ARG (null pointer, root_body out of range, unknown body
 * type, non-finite or non-positive parameter, a colour (rgb, ground_grey, background_rgb) outside [0,1], a
 * negative mesh colour multiplier, degenerate camera, mesh index out of range or non-finite mesh vertex);
 * UNSUPPORTED (width or height outside [8,512], n_bodies outside [1,64], more
 * than 65535 vertices or triangles, tessellation counts outside [3,64]x[1,32]
 * (box [1,16]), or a frame that does not fit the 160 KB of LDS of one
 * compute unit); OOM; DEVICE. */
int pxr_create_scene(const pxr_scene_desc* desc, pxr_scene** out);

/* Free the scene and its device constants (the counterpart of pxr_create_scene; paper section 1: the
 * renderer's state lives on the device for as long as the environments do).  The caller must have
 * synchronised every stream that still renders from it.  NULL is accepted. */
int pxr_destroy_scene(pxr_scene* s);

/* Bind (or with d == NULL / mode NONE, unbind) the distractor that later
 * pxr_render_batch calls fuse into their final per-pixel pass (paper section
 * 2: distractors live inside the renderer).  Host only; launches nothing.
 * Errors: INVALID_ARG (unknown mode, non-finite range, VIDEO with null
 * d_video or n_frames == 0 or alpha outside [0,1]). */
int pxr_apply_distractor(pxr_scene* s, const pxr_distractor_desc* d);

/* Render B environments x S steps = B*S frames (the hot path; paper section 1:
 * one pixel observation per parallel environment per step, on the device).
 *   d_poses  [B,S,K,7] fp32: position xyz, unit quaternion wxyz (body -> world)
 *   d_shapes [B,K,4]   fp32 per-environment shapes, or NULL = the scene's
 *   step0    step index of s = 0 (frame s of the call is step step0 + s; it
 *            keys the generator and selects the video frame)
 *   env0     global index of the batch's first environment (keys the generator,
 *            so a shard renders the same bytes as the whole batch would)
 *   d_frames [B,S,H,W,3] uint8, R,G,B, row-major, written completely
 *   d_ids    [B,S,H,W] uint32 winning triangle id / PXR_ID_GROUND / PXR_ID_BG,
 *            or NULL
 *   hip_stream  hipStream_t to enqueue on; NULL = the default stream
 * Only enqueues and returns: no synchronisation, no host<->device copy, no
 * allocation.  Pose VALUES are not validated.  A triangle with corners on both sides of the near plane
 * z_near is clipped against it (the part in front is drawn); one wholly behind it is not drawn; a vertex
 * in front that projects more than 16384 pixels from the image centre, or a non-finite one, removes its
 * triangles from the frame.
 * Alignment: d_poses, d_frames 4 bytes; d_shapes (16-byte records), d_ids 16 bytes.
 * Errors: INVALID_ARG (null scene/poses/frames, B*S == 0, B*S > 2^31-1,
 * step0 + S or env0 + B overflow, misaligned buffer); DEVICE (launch failure). */
int pxr_render_batch(pxr_scene* s, const float* d_poses, const float* d_shapes, uint32_t B, uint32_t S,
                     uint32_t step0, uint32_t env0, uint8_t* d_frames, uint32_t* d_ids, void* hip_stream);

/* Kinematic tree of the scene's bodies, for callers whose simulator state is joint angles rather than
 * body poses (the paper's loop keeps that state on the device, section 1; this stage turns it into the
 * renderer's input there).  All arrays are host memory, copied by pxr_set_skeleton.
 *   parent[k]  -1: body k is free, its pose is free pose number slot[k] (0 <= slot[k] < n_free), copied
 *              verbatim; otherwise body k hangs on body parent[k] < k by a hinge
 *   slot[k]    hinged body: index of its angle (0 <= slot[k] < n_angles), or -1 = rigidly attached (angle 0)
 *   anchor[k]  hinge position in the parent's frame; axis[k] unit hinge axis (same in both frames);
 *   offset[k]  body centre relative to the hinge, in the body's own frame   (each [n_bodies*3])
 * Pose of a hinged body: q = q_parent (x) (cos(a/2), sin(a/2) axis);
 *   p = (p_parent + R(q_parent) anchor) + R(q) offset,  fp32, R as in the vertex stage.  sin and cos of a/2 are
 *   within 1.25 * 2^-24 of the true values for |a| <= 65536 rad; an angle beyond that or a non-finite one makes
 *   the body's pose, and those of its descendants, NaN (their triangles are not drawn). */
typedef struct {
    uint32_t n_bodies, n_free, n_angles;
    const int32_t* parent;
    const int32_t* slot;
    const float* anchor;
    const float* axis;
    const float* offset;
} pxr_skeleton_desc;

/* Bind (or with k == NULL remove) the scene's skeleton.  Host only; one small allocation and upload.  The
 * caller must have synchronised streams still using the previous skeleton.
 * Errors: INVALID_ARG (null array, n_bodies != the scene's, parent[k] >= k, slot out of range, non-finite
 * entry); UNSUPPORTED (7*n_bodies + 7*n_free + n_angles above 630); OOM; DEVICE. */
int pxr_set_skeleton(pxr_scene* s, const pxr_skeleton_desc* k);

/* Forward kinematics for N frames: d_free_poses [N,n_free,7] and d_angles [N,n_angles] (may be NULL when
 * the count is 0) -> d_poses [N,n_bodies,7] (xyz, wxyz), all fp32 device buffers, 4-byte aligned.  One kernel,
 * four wavefronts per 64 frames; enqueue only.  Errors: INVALID_ARG (no skeleton bound, null or misaligned buffer,
 * N == 0); DEVICE. */
int pxr_pose_batch(pxr_scene* s, const float* d_free_poses, const float* d_angles, uint32_t n_frames,
                   float* d_poses, void* hip_stream);

/* pxr_pose_batch over B*S frames followed by pxr_render_batch on the same stream: joint angles in, frames
 * out, nothing crossing the host.  d_poses [B,S,n_bodies,7] is caller-provided and receives the poses (a
 * learner usually wants them as well); the other arguments are those of the two calls.  Small batches are one
 * launch: the render kernel makes the poses itself, the same bits (pxr_kinematic_info says which). */
int pxr_render_batch_kinematic(pxr_scene* s, const float* d_free_poses, const float* d_angles, const float* d_shapes,
                               uint32_t B, uint32_t S, uint32_t step0, uint32_t env0, float* d_poses,
                               uint8_t* d_frames, uint32_t* d_ids, void* hip_stream);

/* How many kernels pxr_render_batch_kinematic launches for n_frames = B * S frames (buffers that do not overlap):
 * 1 or 2.  Errors: INVALID_ARG (null argument, n_frames == 0, no skeleton bound). */
int pxr_kinematic_info(const pxr_scene* s, uint32_t n_frames, uint32_t* n_launches);

/* pxr_render_batch_kinematic for callers that cannot allocate device memory or provide a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The poses live
 * in a 32 MiB buffer that is part of the library's image on each GPU (held until the process
 * ends) instead of in d_poses, also where the call is one kernel; they are not returned.  The call allocates and frees nothing and only enqueues.
 * Calls on one GPU share that buffer: two calls whose kernels may overlap (different streams without an
 * ordering between them) race; calls on one stream, or ordered by events, are safe.  Nothing carries over
 * from one call to the next.
 * Errors: those of pxr_render_batch_kinematic, and UNSUPPORTED when B * S * n_bodies * 28 bytes exceed
 * 32 MiB (33 554 432); DEVICE if the buffer's address cannot be obtained. */
int pxr_render_batch_kinematic_static(pxr_scene* s, const float* d_free_poses, const float* d_angles,
                                      const float* d_shapes, uint32_t B, uint32_t S, uint32_t step0, uint32_t env0,
                                      uint8_t* d_frames, uint32_t* d_ids, void* hip_stream);

/* ---- frame consumer: the policy's first convolutional layer on the frame stack ----
 * The paper's throughput loop ends every environment step with a forward pass through one convolutional
 * layer on the observations (section 2); it gives no hyper-parameters.  Built here: 3x3 kernel, stride 2, no
 * padding, 32 output channels, the S frames of an environment stacked on the channel axis (channel 3s + c),
 * inputs scaled by 1/255:
 *   out[b,oy,ox,o] = act(bias[o] + sum_{ky,kx,s,c} frames[b,s,2oy+ky,2ox+kx,c]/255 * bf16(w[ky,kx,3s+c,o]))
 * weights rounded to bfloat16 (nearest even) at creation, products and sums in fp32 on the matrix cores,
 * result = fma(sum, 1/255, bias), optional ReLU, rounded to bfloat16 (nearest even). */
typedef struct pxr_conv pxr_conv; /* opaque, owned by the library */
typedef struct {
    uint32_t in_h, in_w, n_stack;  /* frames [B,n_stack,in_h,in_w,3] uint8 */
    uint32_t c_out, kernel, stride; /* must be 32, 3, 2 */
    const float* weights;          /* host [3][3][3*n_stack][32] (height, width, in, out), copied */
    const float* bias;             /* host [32], copied */
    uint32_t relu;                 /* 0 = linear output */
} pxr_conv_desc;

/* Host only.  Errors: INVALID_ARG (null, non-finite weight or bias); UNSUPPORTED (other layer shapes,
 * n_stack outside [1,4], in_h outside [3,512], in_w outside [4,256] or not a multiple of 4); OOM; DEVICE. */
int pxr_conv_create(const pxr_conv_desc* desc, pxr_conv** out);
/* Free a layer made by pxr_conv_create (same passage).  NULL accepted; synchronise streams still using it first. */
int pxr_conv_destroy(pxr_conv* c);

/* d_frames [B,n_stack,in_h,in_w,3] uint8 (what pxr_render_batch writes for S = n_stack) ->
 * d_out [B,out_h,out_w,32] bfloat16 bit patterns, out_h = (in_h-3)/2+1, out_w = (in_w-3)/2+1.
 * Device buffers owned by the caller, d_frames 4-byte and d_out 16-byte aligned.  One kernel, enqueue only.
 * Errors: INVALID_ARG (null, B == 0 or too large, misaligned); DEVICE. */
int pxr_conv_forward(pxr_conv* c, const uint8_t* d_frames, uint32_t B, uint16_t* d_out, void* hip_stream);

/* Facts about a layer (no passage of the paper): output size, output rows per work item, LDS bytes per
 * workgroup, persistent workgroups per launch.  Any pointer may be NULL.  Errors: INVALID_ARG (null layer). */
int pxr_conv_info(const pxr_conv* c, uint32_t* out_h, uint32_t* out_w, uint32_t* band_rows, uint32_t* lds_bytes,
                  uint32_t* n_groups);

/* Tuning knob for benchmarks: output rows per work item and workgroups per launch (0 = default).  The
 * output does not depend on it. */
int pxr_conv_set_tuning(pxr_conv* c, uint32_t band_rows, uint32_t n_groups);

/* ---- renderer and consumer as one step ----
 * The paper's throughput loop (section 2) renders every environment and then runs the conv layer on the
 * frames, every step.  The renderer is bound by vector-ALU issue and the layer by HBM, so this call runs them
 * side by side: the batch is cut into n_chunks runs of environments, chunk c is rendered on the caller's stream
 * and its conv layer follows on a second stream (created here, default priority) while chunk c + 1 is rendered;
 * ordering is by events only, and the caller's stream is made to wait for the last layer before the call
 * returns (enqueue only, no host synchronisation, no allocation).  Frames and features are byte for byte those
 * of pxr_render_batch followed by pxr_conv_forward.  n_chunks = 1 is that serial order, and
 * so is a step whose frames and features take fewer than 2.4 GB (B * (3 * S * H * W + 64 * Ho * Wo) bytes), where
 * overlapping costs more than it gains, unless pxr_pipeline_set_overlap_from says otherwise. */
typedef struct pxr_pipeline pxr_pipeline; /* opaque, owned by the library; borrows the scene and the layer */

/* Host only: one stream and n_chunks + 1 events.  The layer's input size must be the scene's frame size; its
 * n_stack is the S of every step.  Errors: INVALID_ARG (null, n_chunks outside [1,16], sizes differ); OOM; DEVICE. */
int pxr_pipeline_create(pxr_scene* s, pxr_conv* c, uint32_t n_chunks, pxr_pipeline** out);
/* Waits for the second stream, then frees it and the events; scene and layer stay the caller's.  NULL accepted. */
int pxr_pipeline_destroy(pxr_pipeline* p);
/* d_poses [B,S,K,7], d_shapes [B,K,4] or NULL, d_frames [B,S,H,W,3] (written), d_features [B,Ho,Wo,32] bf16
 * (written): arguments, alignment and errors as for pxr_render_batch and pxr_conv_forward.  Steps issued on
 * one pipeline must be ordered among themselves (one stream, or events): they share the second stream. */
int pxr_pipeline_step(pxr_pipeline* p, const float* d_poses, const float* d_shapes, uint32_t B, uint32_t step0,
                      uint32_t env0, uint8_t* d_frames, uint16_t* d_features, void* hip_stream);
/* Bytes of frames and features from which later steps are cut into chunks (host only; 0 = every step, UINT64_MAX = none;
 * no passage of the paper).  The output does not depend on it.  Errors: INVALID_ARG (null). */
int pxr_pipeline_set_overlap_from(pxr_pipeline* p, uint64_t bytes);
/* Into how many chunks a step of B environments is cut (host only; no passage of the paper).  Errors: INVALID_ARG. */
int pxr_pipeline_info(const pxr_pipeline* p, uint32_t B, uint32_t* chunks);

/* ---- a policy's memory: layer norm, linear attention, a gated recurrence, norms and rotation of heads ----
 * The paper's loop (section 2) ends with the first layer of a policy.  What stands behind that layer in a policy that
 * remembers: a normalisation, and a state per environment that each step reads and adds to.  Element types are fp32 and
 * bfloat16; statistics, sums and states are fp32.  All calls only enqueue: no allocation, no synchronisation. */
enum { PXR_F32 = 0, PXR_BF16 = 1 };

/* Layer norm over rows of `width` values:
 *   mean = sum x / width,  rstd = 1 / sqrt(sum (x - mean)^2 / width + eps),  y = (x - mean) * rstd * weight + bias
 * Strides are in elements between the starts of rows; values inside a row are adjacent.  weight and bias are of param_dtype,
 * which is PXR_F32 or dtype. */
typedef struct {
    uint32_t dtype, param_dtype;
    uint64_t n_rows;
    uint32_t width;
    float eps;
    int64_t x_stride; /* rows of x */
    int64_t y_stride; /* rows of y (forward) or of dy (backward) */
    int64_t dx_stride; /* rows of dx (backward) */
} pxr_layer_norm_desc;

/* d_weight, d_bias [width] or NULL (1 and 0); d_mean, d_rstd [n_rows] fp32, written, or NULL where no backward pass
 * follows.  y may be x itself with the same stride.  n_rows == 0 is a call that does nothing.  Values are not validated: a
 * row with a NaN or an infinity comes out as NaN, the other rows are not touched by it.
 * Errors: INVALID_ARG (null, width == 0 or above 2^30, a type that is none, eps negative or not finite, a row stride
 * smaller than the width, a buffer that is not aligned to its elements, n_rows above 2^31-1); DEVICE. */
int pxr_layer_norm_forward(const pxr_layer_norm_desc* d, const void* d_x, const void* d_weight, const void* d_bias,
                           void* d_y, float* d_mean, float* d_rstd, void* hip_stream);

/* Bytes of workspace that pxr_layer_norm_backward needs for this description (host only; may be 0).  Errors: as above. */
int pxr_layer_norm_workspace(const pxr_layer_norm_desc* d, size_t* bytes);

/* Gradients, with g = weight * dy and xh = (x - mean) * rstd from the forward pass' mean and rstd:
 *   dx = rstd * (g - sum g / width - xh * sum(g * xh) / width),  dweight = sum over rows dy * xh,  dbias = sum over rows dy
 * d_dweight, d_dbias [width] of param_dtype, written (not added to), each NULL if not wanted; zeros for n_rows == 0.  dx may
 * be dy or x itself with the same stride.  The sums over rows are taken in an order that depends on the sizes alone: equal
 * inputs give equal bits.  d_workspace: 16-byte aligned, of at least the bytes that pxr_layer_norm_workspace names, used until
 * the call's kernels end.  Errors: as above, and INVALID_ARG (workspace missing, too small or misaligned). */
int pxr_layer_norm_backward(const pxr_layer_norm_desc* d, const void* d_dy, const void* d_x, const float* d_mean,
                            const float* d_rstd, const void* d_weight, void* d_dx, void* d_dweight, void* d_dbias,
                            void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Linear attention with a decay for each head.  Every environment e and head h has a state S [d_key,d_value]:
 *   S_t = (resets[e,t] ? 0 : exp(log_decay[h]) * S_{t-1}) + k_t v_t^T        o_t = scale * S_t^T q_t
 * resets[e,t] != 0 says that step t begins an episode: nothing from before it reaches it, whatever the state held.  The
 * decays are constants of the layer, copied at creation; no gradient is formed for them. */
typedef struct pxr_linear_attention pxr_linear_attention; /* opaque, owned by the library */
typedef struct {
    uint32_t n_heads, d_key, d_value;
    float scale;
    const float* log_decay; /* host [n_heads], natural logarithm of the decay per step: finite, <= 0 */
} pxr_linear_attention_desc;

/* Host only; one small allocation and upload.  Errors: INVALID_ARG (null, n_heads == 0 or above 65535, a size that is 0, a
 * scale that is not finite, a log_decay that is positive or not finite); UNSUPPORTED (d_key or d_value above 256); OOM; DEVICE. */
int pxr_linear_attention_create(const pxr_linear_attention_desc* desc, pxr_linear_attention** out);
/* Free a layer; NULL accepted; synchronise streams still using it first. */
int pxr_linear_attention_destroy(pxr_linear_attention* a);

/* A view [environments, steps, heads, d] of a device buffer: strides in elements, the d values of a head adjacent.  Inputs
 * may have any strides (0 where heads or environments share); views that are written must not overlap themselves. */
typedef struct {
    void* data;
    int64_t env, step, head;
} pxr_tokens;

/* What the layer reads.  d_state [n_envs,n_heads,d_key,d_value] fp32 before the first step, or NULL = zeros. */
typedef struct {
    uint32_t dtype;            /* of q, k, v and of everything that is [.., d]: PXR_F32 or PXR_BF16 */
    uint32_t n_envs, n_steps;
    pxr_tokens q, k, v;
    const uint8_t* d_resets;   /* [n_envs,n_steps] bytes, or NULL = none */
    int64_t resets_env, resets_step; /* its strides */
    const float* d_state;
} pxr_rollout;

/* Bytes of workspace that the forward (backward == 0) or backward pass needs (host only; may be 0).
 * Errors: INVALID_ARG (null, sizes or a type that the calls refuse). */
int pxr_linear_attention_workspace(const pxr_linear_attention* a, uint32_t dtype, uint32_t n_envs, uint32_t n_steps, uint32_t backward,
                                   size_t* bytes);

/* All steps of a rollout at once: out [n_envs,n_steps,n_heads,d_value] of the rollout's type, and the state after the last step
 * in d_state_out [n_envs,n_heads,d_key,d_value] (NULL if not wanted; not the buffer of d_state).  n_steps == 0 passes the
 * state on.  An infinity or NaN in a step's k or v reaches that step and the later ones of the same episode and no others (an
 * infinity may come out as NaN; fp32 values above bfloat16's largest, 3.389e38, count as one, and those below 1e-33 keep fewer
 * digits).  out must not overlap what is read.
 * Errors: INVALID_ARG (null, n_envs == 0, n_envs * n_heads above 2^21, n_steps above 2^31-1, a type that is none, a buffer
 * not aligned to its elements, states that overlap, workspace missing, too small or not 16-byte aligned); DEVICE. */
int pxr_linear_attention_forward(pxr_linear_attention* a, const pxr_rollout* r, const pxr_tokens* out, float* d_state_out,
                                 void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Gradients for the outputs' gradients dout (strides as given) and d_dstate_out (of the state after the last step; NULL = zeros):
 * dq, dk [n_envs,n_steps,n_heads,d_key], dv [.., d_value] of the rollout's type and, unless NULL, d_dstate
 * [n_envs,n_heads,d_key,d_value] fp32, of the state before the first step.  Probabilities and states are computed again, nothing
 * is kept from the forward pass.  What is written must not overlap what is read.  Equal inputs give equal bits.
 * Errors: as for the forward pass. */
int pxr_linear_attention_backward(pxr_linear_attention* a, const pxr_rollout* r, const pxr_tokens* dout,
                                  const float* d_dstate_out, const pxr_tokens* dq, const pxr_tokens* dk, const pxr_tokens* dv,
                                  float* d_dstate, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* One step of every environment: r->n_steps must be 1 (the step strides do not matter), d_state [n_envs,n_heads,d_key,d_value]
 * is updated in place (r->d_state is not read; 4-byte aligned); out must not overlap what is read.  One kernel.
 * Errors: as for the forward pass. */
int pxr_linear_attention_step(pxr_linear_attention* a, const pxr_rollout* r, float* d_state, const pxr_tokens* out, void* hip_stream);

/* A gated linear recurrence.  Every environment e and channel c has a state h:
 *   a_t = 1 / (1 + exp(-gate_t)),   h_t = (resets[e,t] ? 0 : a_t * h_{t-1}) + (coupled ? 1 - a_t : 1) * x_t,   out_t = h_t
 * resets as for linear attention: nothing from before a step that begins an episode reaches it, whatever the state held. */

/* A view [environments, steps, width] of a device buffer: strides in elements, the values of a step adjacent.  Inputs may have any
 * strides (0 where environments or steps share); views that are written must not overlap themselves. */
typedef struct {
    void* data;
    int64_t env, step;
} pxr_steps;

typedef struct {
    uint32_t dtype;            /* of x, gate and of everything that is [.., width]: PXR_F32 or PXR_BF16 */
    uint32_t n_envs, n_steps, width;
    uint32_t coupled;          /* 0 = inputs as they are, 1 = inputs times 1 - a */
    pxr_steps x, gate;
    const uint8_t* d_resets;   /* [n_envs,n_steps] bytes, or NULL = none */
    int64_t resets_env, resets_step; /* its strides */
    const float* d_state;      /* [n_envs,width] fp32 before the first step, or NULL = zeros */
} pxr_gated_rollout;

/* Bytes of workspace that the forward (backward == 0) or backward pass needs (host only; may be 0).
 * Errors: INVALID_ARG (null, sizes that the calls refuse). */
int pxr_gated_recurrence_workspace(uint32_t n_envs, uint32_t n_steps, uint32_t width, uint32_t backward, size_t* bytes);

/* All steps of a rollout at once: out [n_envs,n_steps,width] of the rollout's type, and the state after the last step in d_state_out
 * [n_envs,width] fp32 (NULL if not wanted; not the buffer of d_state).  n_steps == 0 passes the state on.  An infinity or NaN in a step's
 * x or gate reaches that step and later ones of the same environment, channel and episode and nothing else (an infinity may come out as NaN); where coupled is 0, the gate
 * of a step that begins an episode is not looked at, and its gradient is 0 (where those of the outputs are finite).
 * What is written must not overlap what is read.  Equal inputs give equal bits.
 * Errors: INVALID_ARG (null, n_envs or width == 0, n_envs * ceil(width / 64) * ceil(n_steps / 128) above 2^22, n_steps above 2^31-1, a type
 * that is none, coupled above 1, a buffer not aligned to its elements, states that overlap, a view that is written and has values in common with another of
 * the same strides, workspace missing, too small or not 16-byte aligned); DEVICE. */
int pxr_gated_recurrence_forward(const pxr_gated_rollout* r, const pxr_steps* out, float* d_state_out, void* d_workspace,
                                 size_t workspace_bytes, void* hip_stream);

/* Gradients for the outputs' gradients dout and d_dstate_out (of the state after the last step; NULL = zeros): dx, dgate
 * [n_envs,n_steps,width] of the rollout's type and, unless NULL, d_dstate [n_envs,width] fp32, of the state before the first step.  States are
 * computed again in fp32, nothing is kept from the forward pass.  An infinity or NaN in dout reaches that step and earlier ones of the same
 * environment, channel and episode.  What is written must not overlap what is read, or itself.  Equal inputs give equal bits.
 * Errors: as for the forward pass. */
int pxr_gated_recurrence_backward(const pxr_gated_rollout* r, const pxr_steps* dout, const float* d_dstate_out, const pxr_steps* dx,
                                  const pxr_steps* dgate, float* d_dstate, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* One step of every environment: r->n_steps must be 1 (the step strides do not matter), d_state [n_envs,width] is updated in place
 * (r->d_state is not read); out must not overlap what is read, but may be x or gate itself.  One kernel.  Errors: as for the forward pass. */
int pxr_gated_recurrence_step(const pxr_gated_rollout* r, float* d_state, const pxr_steps* out, void* hip_stream);

/* Norms of queries and keys for each head, with the rotation by a step's position in the same pass: what stands before attention
 * where queries and keys grow together or the distance between steps should count.  For a head's values x [d_head] of a step at position p:
 *   y = x / sqrt(sum x^2 / d_head + eps) * weight
 *   the pairs (y_i, y_{i + d_rotary/2}), i < d_rotary/2, are turned by p * frequencies[i]:  (u, v) -> (u cos - v sin, v cos + u sin)
 * Values from d_rotary on stay as they are.  Angles keep 2^-22 of a turn up to positions of 2^31. */
typedef struct pxr_head_norm pxr_head_norm; /* opaque, owned by the library */
typedef struct {
    uint32_t d_head, d_rotary;  /* d_rotary: even, at most d_head; 0 = no rotation */
    const double* frequencies;  /* host [d_rotary/2], radians a position: finite; copied */
    float eps;
} pxr_head_norm_desc;

/* Host only; one small allocation and upload.  Errors: INVALID_ARG (null, d_head == 0, d_rotary odd or above d_head, a frequency that
 * is not finite or above 2^20, eps negative or not finite); UNSUPPORTED (d_head above 256); OOM; DEVICE. */
int pxr_head_norm_create(const pxr_head_norm_desc* desc, pxr_head_norm** out);
/* Free a layer; NULL accepted; synchronise streams still using it first. */
int pxr_head_norm_destroy(pxr_head_norm* n);

/* What the layer reads.  Single steps are n_steps == 1. */
typedef struct {
    uint32_t dtype, param_dtype;     /* of the heads; of the weights: PXR_F32 or dtype */
    uint32_t n_envs, n_steps;
    uint32_t n_heads, n_key_heads;   /* either may be 0 */
    pxr_tokens q, k;                 /* [n_envs,n_steps,n_heads,d_head], [n_envs,n_steps,n_key_heads,d_head] */
    const void *d_q_weight, *d_k_weight; /* [d_head] or NULL = 1 */
    const void* d_positions;         /* [n_envs,n_steps] signed integers of position_bits bits, or NULL: step t is at first + t */
    uint32_t position_bits;          /* 32 or 64 */
    int64_t positions_env, positions_step; /* strides, in positions */
    int64_t first;
} pxr_heads;

/* The normalised and turned heads to q_out and k_out (NULL where there are no such heads), views of the layout of q and k; either may be its input
 * itself with the same strides.  Sums of squares are fp32.  A head with a NaN or an infinity comes out with NaN in it, the other heads are not touched by it.
 * One kernel.  Errors: INVALID_ARG (null, a type that is none, position_bits that is neither, n_envs * n_steps above 2^31-1, n_heads or n_key_heads above 65535, a
 * buffer not aligned to its elements, heads that are written and have values in common with others of the same strides than their own inputs); DEVICE. */
int pxr_head_norm_forward(pxr_head_norm* n, const pxr_heads* r, const pxr_tokens* q_out, const pxr_tokens* k_out, void* hip_stream);

/* Bytes of workspace that the backward pass needs where it forms a weight's gradient (host only).  Errors: as above (buffers are not looked at). */
int pxr_head_norm_workspace(const pxr_head_norm* n, const pxr_heads* r, size_t* bytes);

/* Gradients for those of the outputs, dq_out and dk_out: dq, dk, and the weights' d_dq_weight, d_dk_weight [d_head] of param_dtype, written (not
 * added to), each NULL if not wanted; zeros where there are no such heads.  dq may be q or dq_out itself with the same strides, dk likewise.  Statistics and
 * angles are computed again.  Equal inputs give equal bits.  d_workspace: 16-byte aligned, used until the call's kernels end.  Errors: as above, and INVALID_ARG
 * (workspace missing, too small or misaligned). */
int pxr_head_norm_backward(pxr_head_norm* n, const pxr_heads* r, const pxr_tokens* dq_out, const pxr_tokens* dk_out, const pxr_tokens* dq, const pxr_tokens* dk,
                           void* d_dq_weight, void* d_dk_weight, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* ---- a learner's update with its singular values pushed towards one ----
 * For what an optimiser is about to add to a weight matrix (a gradient, its momentum): every direction of the update counts alike.  Of a
 * matrix x [rows,cols]; where it has more rows than columns, of its transpose:
 *   X = x / (|x| + eps), |x| the Frobenius norm;   n_steps times  X <- a X + (b A + c A^2) X,  A = X X^T,  with (a, b, c) = coefficients of that step
 * A singular value t goes through t <- a t + b t^3 + c t^5.  Several matrices of one size go together. */
typedef struct {
    uint32_t dtype;                 /* of x and of the result: PXR_F32 or PXR_BF16 */
    uint32_t n_matrices, rows, cols;
    int64_t x_matrix, x_row;        /* strides of x in elements; the values of a row are adjacent */
    int64_t out_matrix, out_row;    /* of the result */
    uint32_t n_steps;
    const float* coefficients;      /* host [n_steps][3], read during the call */
    float eps;
} pxr_orthogonalise_desc;

/* Bytes of workspace that pxr_orthogonalise needs for this description (host only; may be 0).  Errors: as for the call (buffers are not looked at). */
int pxr_orthogonalise_workspace(const pxr_orthogonalise_desc* d, size_t* bytes);

/* The result in d_out, which may be d_x itself with the same strides.  Products and sums keep 22 bits and more (fp32's, but for a few roundings of 2^-23); values below 2^-38 of the
 * bound that the coefficients set for the singular values (1 before the first step) are zeros, so an update whose norm is far below eps comes out as zeros.  Where the smaller of rows and cols is at
 * most 32 and the larger above 320, products, sums and values between the steps are fp64: no value is lost so, and such an update comes out small.  Directions that a matrix does not have are made of those roundings, 2^-23 or 2^-53, which
 * grow with its small singular values: after some 13 steps of 3.4, or 30, they are as large as the others.  A matrix
 * with a NaN or an infinity comes out as NaN, the others are not touched by it.  n_matrices == 0 is a call that does nothing.  Equal inputs give equal bits.
 * d_workspace: 16-byte aligned, used until the call's kernels end.
 * Errors: INVALID_ARG (null, rows or cols == 0, a type that is none, n_steps outside [1,64], a coefficient that is not finite, steps under which a
 * singular value may pass 2^20 or grow by more than 10^12, eps negative or not finite, a row stride smaller than cols, matrices of the result that overlap, a result that has values
 * in common with x of the same strides and is not x itself, n_matrices above 65535, a buffer not aligned to its elements, workspace missing, too small or not 16-byte aligned); UNSUPPORTED (the smaller of rows and cols above 2^15, the larger above 2^28, rows * cols above 2^32);
 * DEVICE. */
int pxr_orthogonalise(const pxr_orthogonalise_desc* d, const void* d_x, void* d_out, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Scene facts for callers and tests (sizes of what pxr_create_scene built; no passage of the paper): total
 * template vertices and triangles, dynamic LDS bytes per frame workgroup, threads per workgroup.  Any out
 * pointer may be NULL.  block_threads is that of launches which fill the device; smaller ones may take another.
 * Errors: INVALID_ARG (null scene). */
int pxr_scene_info(const pxr_scene* s, uint32_t* n_verts, uint32_t* n_tris, uint32_t* lds_bytes,
                   uint32_t* block_threads);

/* Override the threads per frame workgroup (256, 512, 768 or 1024); 0 restores the
 * default.  A tuning knob for benchmarks; output does not depend on it. */
int pxr_set_block_threads(pxr_scene* s, uint32_t threads);

/* Measurement aid (synchronous, allocates 2 GiB for the duration of the call): the rates this GPU sustains
 * on a dependent-free fp32 FMA loop and on a 24-bit integer multiply-add loop (both in T lane-operations/s,
 * 32 waves per compute unit), the read+write bandwidth of a plain 1 GiB device-to-device copy and the
 * bandwidths of a 2 GiB read-only and a 2 GiB write-only stream (GB/s; HBM does not give both directions
 * the same rate).  Lets a roofline fraction be quoted against the machine as it runs.  Any pointer may be
 * NULL.  Errors: OOM, DEVICE. */
int pxr_measure_peaks(double* fma_tlaneops, double* imad_tlaneops, double* copy_gbs, double* read_gbs, double* write_gbs);

/* Verification aid (synchronous, a few tens of milliseconds): the render kernel replaces two operations whose
 * results decide integers by shorter instruction sequences - 1/x by the hardware estimate plus one fused
 * Newton step, (int)floorf(x) by one converting instruction.  This call compares each with the plain form on
 * the current device for EVERY 32-bit pattern in its domain (x in [2^-100, 2^100]; every x that is not NaN)
 * and writes to the host array counts[4]: reciprocal mismatches, floor mismatches, patterns checked by the
 * first and by the second comparison.  Both mismatch counts must be 0 on a device the library supports.
 * Errors: INVALID_ARG (null), OOM, DEVICE. */
int pxr_selftest_arithmetic(uint64_t* counts);

/* Host-only introspection: run the scene builder of pxr_create_scene without
 * touching a device and copy out its tables, so that the tessellation and the
 * camera constants can be checked on a machine without a GPU.  Any output
 * pointer may be NULL.  Same validation errors as pxr_create_scene.
 *   vtmpl     [V*4] ux,uy,uz and a word holding body<<2 | (s+1)
 *   tri_idx   [T*2] v0 | v1<<16 ,  v2 | body<<16
 *   tri_shade [T*4] unit normal in the body frame, colour multiplier
 *   cxcy      [W+H] ray slopes of the pixel-centre columns, then rows
 *   consts    [16]  right[3], up[3], forward[3], focal, ground shade[2], light[3], LDS bytes
 *   pair_tbl  [P*3] binning table: q0 | q1<<16, q2 | q3<<16, triA | triB<<16 (two triangles sharing the
 *             edge q0-q2; a lone triangle has q3 = q2 and triB = 0xFFFF); P is returned in n_pairs */
int pxr_host_tables(const pxr_scene_desc* desc, uint32_t* n_verts, uint32_t* n_tris, float* vtmpl, uint32_t* tri_idx,
                    float* tri_shade, float* cxcy, float* consts, uint32_t* n_pairs, uint32_t* pair_tbl);

/* Reason for the last failure on this thread; valid until the next call on it.  (Error reporting of this
 * interface; no passage of the paper.) */
const char* pxr_last_error(void);

#ifdef __cplusplus
}
#endif
#endif
